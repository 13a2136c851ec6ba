// Attention with a sliding window, first tokens that stay visible (sinks) and
// a learned relative position bias, forward and backward, on CDNA4 matrix
// cores, for bf16 and fp32 tensors and head dimensions up to 128.
//
//   x_ij = (scale q_i.k_j + bias[h, bucket(j - i)]) log2(e)
//   j visible to i:  j < len, i < len and (-left <= j - i <= right or
//                    (j < sinks and (not causal or j <= i)))
//   P_ij = 2^(x_ij - m_i - l_i) over the visible j;  o_i = sum_j P_ij v_j
//   D_i = do_i.o_i;  dS_ij = P_ij (do_i.v_j - D_i)
//   dq_i = scale sum_j dS_ij k_j;  dk_j = scale sum_i dS_ij q_i
//   dv_j = sum_i P_ij do_i;  dbias[h, c] = sum of dS_ij with bucket(j - i) = c
//
// One pass over the visible key blocks per block of 128 queries with a running
// reference m and sum (forward, dq, dbias), one over the visible query blocks
// per block of 128 keys (dk, dv); blocks that no query sees are not visited.
// The score blocks come out of the matrix cores with one query (or one key)
// per lane column, as in attn_flash_kernels.h, whose fragment and copy
// helpers the bf16 kernels use; masks cost vector work only in blocks that
// straddle an edge of the window, the sequence or the sinks.
//
// Bias: the distances of less than `far` tokens have a table in LDS (the
// bias of distance e - off at entry e); a block whose distances are all at
// least that takes one value.  Its gradient: each wave adds the dS of a near
// block to a table of its own by distance (no two lanes of an instruction meet:
// every sum has a fixed order); far blocks add up in registers.  The tables are summed by buckets
// when the workgroup ends, and over workgroups by the next kernel (dk and dv).
//
// Exponents are taken of score differences, and D is formed by the same chain of
// matrix instructions as do.v: where a row sees one token only, its probability
// is exactly one and dS exactly zero.
//
// us, forward / dq / dk and dv: 32 heads of 128, s 2048, causal, 32 buckets: 77 /
// 104 / 114; 32 and 8 heads of 128, s 8192, window 1024: 197 / 263 / 393; 16 heads
// of 64, 8 sequences of 512, both directions, 32 buckets: 26 / 41 / 29.  The matrix cores are busy
// for 26 to 43 % of the cycles, vector instructions issue in 18 to 32 % of a wave's
// cycles and LDS ones in 4 to 9 %: no unit is full.  The rest goes to waits (for LDS data,
// of which transposed reads come at half the rate, and for tiles at the barriers)
// that one or two waves a SIMD do not cover; dk and dv at 128 columns have one
// (two, with half of the columns each, read LDS twice: 518).
// Blocks of 128 rows on one side keep the other side's reads from memory small;
// grids that would leave compute units empty split further (attn_op.h).
#pragma once

#include "attn_flash_kernels.h"
#include "attn_op.h"

namespace {

// Element r of a 32x32 block: row 4 (lane / 32) + kofs(r).
__device__ __forceinline__ constexpr int row_of(int r) { return 8 * (r >> 2) + (r & 3); }
__device__ __forceinline__ bool wave_uniform(bool c) { return __builtin_amdgcn_readfirstlane((int)c) != 0; }

// What the kernels need of a tensor type: tiles of 64 rows in LDS, operands
// that stay in registers, the two kinds of products, stores.
template <int HD_>
struct TileB16 {
  using E = bf16;
  using A = Attn<HD_, false>;
  static constexpr int HD = HD_, TILE = A::TILE64;
  static constexpr bool DIRECT = false, REST = true;
  // waves a SIMD of the kernels over queries and keys
  static constexpr int WAVES = 2, KWAVES = HD > 96 ? 1 : 2;
  static constexpr int FWAVES = 1, QWAVES = 1, DWAVES = 1;  // of the kernels of 32 rows, at least
  using Rows = bf16x8[HD / 16];
  struct Offs {
    typename A::RowOffs ro;
    typename A::TrOffs to;
    __device__ __forceinline__ void init(int lane) {
      ro.init(lane);
      to.init(lane);
    }
  };
  struct Src {
    i32x4 rs;
    long ld;
    __device__ __forceinline__ void set(const E* base, long ld_, int rows) {
      ld = ld_;
      rs = make_rsrc(base, rows > 0 ? 2L * ((long)(rows - 1) * ld_ + HD) : 0);
    }
  };
  static __device__ __forceinline__ void copy(char* tile, const Src& s, int wave, int lane, int row0, int nrows, int d) {
    A::template load_tile<64>(s.rs, tile, wave, lane, s.ld, row0, nrows, d);
  }
  // 32 rows by one wave alone into an area of its own (OWN bytes), and what the products read of them
  static constexpr int OWN = TILE / 2;
  using Block = const char*;
  static __device__ __forceinline__ Block block(const Src&, const char* own, int, int, int) { return own; }
  static __device__ __forceinline__ void copy_own(char* tile, const Src& s, int lane, int row0, int nrows, int d) {
#pragma unroll
    for (int v = 0; v < 4; ++v) A::template load_tile<32>(s.rs, tile, v, lane, s.ld, row0, nrows, d);
  }
  static __device__ __forceinline__ void own_landed() { A::own_copies_landed(); }
  static __device__ __forceinline__ void own_read() { A::own_reads_done(); }
  // n (32 or 64) floats into a 1 KB area; issued by one wave
  static __device__ __forceinline__ void vec(char* dst, const float* src, int lane, int n = 64) {
    A::load_vec64(make_rsrc(src, 4 * n), dst, lane, 0, n);
  }
  static __device__ __forceinline__ const float* vec_of(const char* own, const float*) { return (const float*)own; }
  static __device__ __forceinline__ void rows(Rows& f, const E* base, long ld, int row, int nrows, int lane, int d) {
    A::load_stationary(f, base, ld, row, nrows, lane, d);
  }
  // a0 += block b0 of tile t0 times s0, a1 += block b1 of tile t1 times s1
  static __device__ __forceinline__ void score2(f32x16& a0, const char* t0, int b0, const Rows& s0, f32x16& a1,
                                                const char* t1, int b1, const Rows& s1, const Offs& o, int) {
    A::template two_chains<2>(a0, t0, b0, s0, a1, t1, b1, s1, o.ro);
  }
  static __device__ __forceinline__ void score1(f32x16& a, const char* t, const Rows& s, const Offs& o, int) {
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks) a = A::mfma(A::rd_row(t, o.ro, 0, ks), s[ks], a);
  }
  // a += rows x times rows y, both from registers
  static __device__ __forceinline__ void dot(f32x16& a, const Rows& x, const Rows& y) {
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks) a = A::mfma(x[ks], y[ks], a);
  }
  // acc += (32 rows j of the tile)^T times the block p, which is rounded to bf16 for
  // that; FINE: and times what the rounding drops.
  template <bool FINE>
  static __device__ __forceinline__ void outer(f32x16 (&acc)[HD / 32], const char* tile, int j, const f32x16& p,
                                               const Offs& o, int) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const bf16x8 pf = A::pack_half(p, hf);
      bf16x8 rest;
      if constexpr (FINE) {
#pragma unroll
        for (int e = 0; e < 8; ++e) rest[e] = (bf16)(p[8 * hf + e] - (float)pf[e]);
      }
#pragma unroll
      for (int b = 0; b < HD / 32; ++b) {
        const bf16x8 t = A::rd_tr(tile, o.to, b, 2 * j + hf);
        acc[b] = A::mfma(t, pf, acc[b]);
        if constexpr (FINE) acc[b] = A::mfma(t, rest, acc[b]);
      }
    }
  }
  static __device__ __forceinline__ void store(const f32x16 (&acc)[HD / 32], char* t, E* base, long ld, int row0,
                                               int nrows, int lane, float mul, int d) {
    A::store_rows_lds(acc, t, base, ld, row0, nrows, lane, mul, d);
  }
  // columns 32 b.. alone
  static __device__ __forceinline__ void store_cols(const f32x16& acc, E* base, long ld, int row0, int nrows, int b,
                                                    int lane, float mul, int d) {
    A::store_block(acc, base, ld, row0 + (lane & 31), nrows, b, lane, mul, d);
  }
};

// fp32: no tiles.  A matrix instruction of 32x32x2 takes 64 cycles for the 4 bytes a
// lane of either operand, so the products read theirs from the caches as they go;
// no barrier ties the waves of a workgroup, and with 32 rows a workgroup (the only
// form) what no pair of a block of 32 x 32 needs is not computed.  us of a training
// step (tiles of 64 rows in LDS, 128 rows a workgroup, against this): 4 sequences
// of 955, 16 / 4 heads of 96, window 6, 16 sinks: 528, 274; 2 of 814, 11 heads of 128,
// both directions, a bias: 774, 562 (matrix instructions run in 58 % of the
// cycles of the busy compute units; most of the rest is vector work next to one wave a SIMD and
// the ends of the workgroups).
template <int HD_>
struct TileF32 {
  using E = float;
  static constexpr int HD = HD_;
  static constexpr bool DIRECT = true, REST = false;
  static constexpr int OWN = 0;
  static constexpr int FWAVES = 2, QWAVES = HD > 96 ? 1 : 2, DWAVES = HD > 64 ? 1 : 2;
  // of every 8 columns the halves of a wave hold 4 each
  using Rows = float[HD / 2];
  struct Offs {
    __device__ __forceinline__ void init(int) {}
  };
  struct Src {
    const E* p;
    long ld;
    __device__ __forceinline__ void set(const E* base, long ld_, int) {
      p = base;
      ld = ld_;
    }
  };
  // 32 rows: rows behind the last one and columns behind the head stand for
  // others of the tensor, whose products meet zeros or are not stored.
  struct Block {
    const char* p;  // first row
    unsigned ld;    // bytes
    int last, d;
    __device__ __forceinline__ float4 row4(int lane, int i) const {
      const char* const at = p + 32 * min(i, d / 8 - 1);
      return *(const float4*)(at + (min(lane & 31, last) * ld + 16u * (lane >> 5)));
    }
    __device__ __forceinline__ float at(int lane, int r, int b) const {
      const unsigned c = min(32 * b + (lane & 31), d - 1);
      return *(const float*)(p + (min(4 * (lane >> 5) + row_of(r), last) * ld + 4 * c));
    }
  };
  static __device__ __forceinline__ Block block(const Src& s, const char*, int row0, int nrows, int d) {
    return {(const char*)(s.p + (long)row0 * s.ld), (unsigned)(4 * s.ld), nrows - 1 - row0, d};
  }
  static __device__ __forceinline__ void copy_own(char*, const Src&, int, int, int, int) {}
  static __device__ __forceinline__ void own_landed() {}
  static __device__ __forceinline__ void own_read() {}
  static __device__ __forceinline__ void vec(char*, const float*, int, int) {}
  static __device__ __forceinline__ const float* vec_of(const char*, const float* src) { return src; }
  static __device__ __forceinline__ void rows(Rows& f, const E* base, long ld, int row, int nrows, int lane, int d) {
#pragma unroll
    for (int k = 0; k < HD / 2; k += 4) {
      const int c = 2 * k + 4 * (lane >> 5);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (row < nrows && c < d) v = *(const float4*)(base + (long)row * ld + c);
      f[k] = v.x;
      f[k + 1] = v.y;
      f[k + 2] = v.z;
      f[k + 3] = v.w;
    }
  }
  static __device__ __forceinline__ f32x16 mfma(float a, float b, const f32x16& c) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ void mfma4(f32x16& a, const float4& u, const float* s) {
    a = mfma(u.x, s[0], a);
    a = mfma(u.y, s[1], a);
    a = mfma(u.z, s[2], a);
    a = mfma(u.w, s[3], a);
  }
  // Loads run AHEAD of the products that take them (the compiler, left to itself,
  // issues each just before).
  static constexpr int AHEAD = HD / 8 < 4 ? HD / 8 : 4;
  static __device__ __forceinline__ void score1(f32x16& a, const Block& t, const Rows& s, const Offs&, int lane) {
    float4 u[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) u[i] = t.row4(lane, i);
#pragma unroll
    for (int i = 0; i < HD / 8; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      const float4 x = u[i % AHEAD];
      if (i + AHEAD < HD / 8) u[i % AHEAD] = t.row4(lane, i + AHEAD);
      mfma4(a, x, s + 4 * i);
    }
  }
  static __device__ __forceinline__ void score2(f32x16& a0, const Block& t0, int, const Rows& s0, f32x16& a1,
                                                const Block& t1, int, const Rows& s1, const Offs& o, int lane) {
    score1(a0, t0, s0, o, lane);
    score1(a1, t1, s1, o, lane);
  }
  static __device__ __forceinline__ void dot(f32x16& a, const Rows& x, const Rows& y) {
#pragma unroll
    for (int k = 0; k < HD / 2; ++k) a = mfma(x[k], y[k], a);
  }
  template <bool>
  static __device__ __forceinline__ void outer(f32x16 (&acc)[HD / 32], const Block& t, int, const f32x16& p, const Offs&,
                                               int lane) {
    constexpr int NB = HD / 32, N = 16 * NB, A = 16;
    float u[A];
#pragma unroll
    for (int i = 0; i < A; ++i) u[i] = t.at(lane, i / NB, i % NB);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);
      const float x = u[i % A];
      if (i + A < N) u[i % A] = t.at(lane, (i + A) / NB, (i + A) % NB);
      acc[i % NB] = mfma(x, p[i / NB], acc[i % NB]);
    }
  }
  static __device__ __forceinline__ void store_cols(const f32x16& acc, E* base, long ld, int row0, int nrows, int b,
                                                    int lane, float mul, int d) {
    const int row = row0 + (lane & 31);
    if (row >= nrows) return;
    E* p = base + (long)row * ld + 32 * b + 4 * (lane >> 5);
#pragma unroll
    for (int g = 0; g < 4; ++g)
      if (32 * b + 8 * g + 4 * (lane >> 5) < d)
        *(float4*)(p + 8 * g) =
            make_float4(acc[4 * g] * mul, acc[4 * g + 1] * mul, acc[4 * g + 2] * mul, acc[4 * g + 3] * mul);
  }
};

template <class T, bool BIAS>
struct AttnOp {
  using E = typename T::E;
  using Rows = typename T::Rows;
  using Offs = typename T::Offs;
  using Src = typename T::Src;
  using Block = typename T::Block;
  static constexpr int HD = T::HD, NB = HD / 32;
  static constexpr float kNone = -3.402823466e38f;

  static __device__ __forceinline__ void zero(f32x16& a) {
#pragma unroll
    for (int r = 0; r < 16; ++r) a[r] = 0.f;
  }
  static __device__ __forceinline__ const E* base(const AttnOpView& v, int b, int h) {
    return (const E*)v.p + (long)b * v.b + (long)h * v.h;
  }
  static __device__ __forceinline__ E* out(const AttnOpView& v, int b, int h) {
    return (E*)v.p + (long)b * v.b + (long)h * v.h;
  }
  static __device__ __forceinline__ int length(const AttnOpArgs& p, int b) {
    if (!p.lengths) return p.s;
    return __builtin_amdgcn_readfirstlane(max(0, min(p.lengths[b], p.s)));
  }

  // -- bias table --------------------------------------------------------------
  // Entry e holds the bias (base 2) of distance j - i = e - off.  A near block of
  // 32 queries and 64 keys reaches at most 94 tokens beyond `far` (and 67 beyond
  // a causal query, where the sums by distance count in).
  static __host__ __device__ __forceinline__ int table_off(const AttnOpArgs& p) { return p.far + 96; }
  static __host__ __device__ __forceinline__ int table_len(const AttnOpArgs& p) {
    return p.far + 96 + (p.causal ? 96 : p.far + 96);
  }
  static __device__ __forceinline__ int bucket_of(const AttnOpArgs& p, int rel) {
    const int side = p.causal ? p.buckets : p.buckets / 2;
    const int n = p.causal ? max(-rel, 0) : abs(rel);
    const int c = n >= p.far ? side - 1 : p.bucket[n];
    return !p.causal && rel > 0 ? c + side : c;
  }
  static __device__ __forceinline__ float bias_at(const AttnOpArgs& p, int h, int rel) {
    const long i = (long)h * p.buckets + bucket_of(p, rel);
    const float v = p.bias_f32 ? ((const float*)p.bias)[i] : (float)((const bf16*)p.bias)[i];
    // finite values stay finite in base 2 (a row of lowest values is uniform)
    const float x = v * 1.4426950408889634f;
    return fabsf(v) <= 3.402823466e38f ? fminf(fmaxf(x, -1.7e38f), 1.7e38f) : x;
  }
  static __device__ __forceinline__ void fill_table(const AttnOpArgs& p, int h, float* table) {
    for (int e = threadIdx.x; e < table_len(p); e += blockDim.x) table[e] = bias_at(p, h, e - table_off(p));
  }
  // Adds a block (lane column = query, elements = keys) to a table by distance
  // whose entry `to` belongs to this lane's query and key row 4 (lane / 32).
  // With b = row_of(r) % 16, lane i of a row of 16 holds the distance that lane
  // i - b holds at row 0, so each element is shifted by b lanes (an addition
  // with a DPP operand) into the sum of its distance: to[0], to[16] for what
  // leaves the row of lanes and for rows 16 and on, to[32] for both.  30
  // additions and three LDS atomics a half for 16 elements (us, dq of 40 heads of 128, s
  // 4096, window 2048, 64 buckets: 334, against 639 with sixteen atomics).
  template <int R>
  static __device__ __forceinline__ void shift_in(float& stays, float& leaves, const f32x16& x) {
    constexpr int b = row_of(R) % 16;
    const int v = __float_as_int(x[R]);
    if constexpr (b == 0) {
      stays += x[R];
    } else {
      stays += __int_as_float(__builtin_amdgcn_update_dpp(0, v, 0x100 + b, 0xf, 0xf, true));         // lane i + b
      leaves += __int_as_float(__builtin_amdgcn_update_dpp(0, v, 0x110 + 16 - b, 0xf, 0xf, true));  // lane i + b - 16
    }
  }
  static __device__ __forceinline__ void add_diagonals(float* to, const f32x16& x, int lane) {
    float s0 = 0.f, s1 = 0.f, s2 = 0.f;
    shift_in<0>(s0, s1, x);
    shift_in<1>(s0, s1, x);
    shift_in<2>(s0, s1, x);
    shift_in<3>(s0, s1, x);
    shift_in<4>(s0, s1, x);
    shift_in<5>(s0, s1, x);
    shift_in<6>(s0, s1, x);
    shift_in<7>(s0, s1, x);
    shift_in<8>(s1, s2, x);
    shift_in<9>(s1, s2, x);
    shift_in<10>(s1, s2, x);
    shift_in<11>(s1, s2, x);
    shift_in<12>(s1, s2, x);
    shift_in<13>(s1, s2, x);
    shift_in<14>(s1, s2, x);
    shift_in<15>(s1, s2, x);
    // one half of the wave after the other: no two lanes of an instruction meet
#pragma unroll
    for (int half = 0; half < 2; ++half)
      if ((lane >> 5) == half) {
        __hip_atomic_fetch_add(to, s0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        __hip_atomic_fetch_add(to + 16, s1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        __hip_atomic_fetch_add(to + 32, s2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      }
  }

  // x = sc sl2 + bias of 32 keys from k (element r, this lane: key k + 4 hh + row_of(r))
  // and this lane's query.
  // dir = 1: lane column = query, elements = keys; -1: the other way round.
  template <int DIR>
  static __device__ __forceinline__ void add_bias(f32x16& sc, const float* table, int e, float c, bool near,
                                                  const AttnOpArgs& p) {
    if (near) {
      const float* t = table + e;
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = fmaf(sc[r], p.sl2, t[DIR * row_of(r)]);
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = fmaf(sc[r], p.sl2, c);
    }
  }

  // -- which blocks a query or key block visits -----------------------------------
  struct Steps {  // tiles [0, n1) and then [t0, t0 + n - n1)
    int n1, t0, n;
    __device__ __forceinline__ int tile(int it) const { return it < n1 ? it : it - n1 + t0; }
  };
  // key tiles of NK for the queries [q0, q1]
  template <int NK>
  static __device__ __forceinline__ Steps key_steps(const AttnOpArgs& p, int q0, int q1, int len) {
    Steps s;
    q1 = min(q1, len - 1);
    if (q1 < q0) return {0, 0, 0};
    const int lo = max(0, q0 - p.left), hi = min((long)len - 1, (long)q1 + p.right);
    const int ns = p.causal ? min(p.sinks, q1 + 1) : min(p.sinks, len);
    const int nts = (ns + NK - 1) / NK;
    s.t0 = lo / NK;
    s.n1 = min(nts, s.t0);
    s.n = s.n1 + max(hi / NK, nts - 1) - s.t0 + 1;
    return s;
  }
  // For 32 queries from q0 and NK keys from k0: whether none / all pairs are visible.
  template <int NK>
  static __device__ __forceinline__ bool none_visible(const AttnOpArgs& p, int q0, int k0, int len) {
    if (q0 >= len || k0 >= len) return true;
    if (p.causal && k0 > q0 + 31) return true;
    if (k0 < p.sinks) return false;
    return k0 - (q0 + 31) > p.right || k0 + NK - 1 - q0 < -p.left;
  }
  template <int NQ, int NK>
  static __device__ __forceinline__ bool all_visible(const AttnOpArgs& p, int q0, int k0, int len) {
    if (q0 + NQ > len || k0 + NK > len) return false;
    if (k0 + NK - 1 - q0 <= p.right && k0 - (q0 + NQ - 1) >= -p.left) return true;
    return k0 + NK <= p.sinks && (!p.causal || k0 + NK - 1 <= q0);
  }

  // Key blocks visit one of three sets of pairs: those of the windows, those that
  // are visible to a sink alone, or both.
  enum { WINDOW, SINK, BOTH };
  template <int MODE>
  static __device__ __forceinline__ bool none_of(const AttnOpArgs& p, int q0, int k0, int len) {
    if (q0 >= len || k0 >= len || (p.causal && k0 > q0 + 31)) return true;
    const bool window = k0 - (q0 + 31) <= p.right && k0 + 31 - q0 >= -p.left;
    const bool sink = k0 < p.sinks && (k0 - (q0 + 31) < -p.left || k0 + 31 - q0 > p.right);
    return MODE == WINDOW ? !window : MODE == SINK ? !sink : !window && !sink;
  }
  template <int MODE>
  static __device__ __forceinline__ bool all_of(const AttnOpArgs& p, int q0, int k0, int len) {
    if (q0 + 32 > len || k0 + 32 > len) return false;
    const bool window = k0 + 31 - q0 <= p.right && k0 - (q0 + 31) >= -p.left;
    if (MODE != SINK && window) return true;
    if (MODE == WINDOW || k0 + 32 > p.sinks || (p.causal && k0 + 31 > q0)) return false;
    return MODE == BOTH || k0 + 31 - q0 < -p.left || k0 - (q0 + 31) > p.right;
  }
  // Lane column = key kk, elements = the queries q + 4 hh + row_of(r): others become 0.
  template <int MODE>
  static __device__ __forceinline__ void mask_queries(f32x16& sc, int q, int kk, int lane, int len, const AttnOpArgs& p) {
    const int at = q + 4 * (lane >> 5);
    const bool sink = MODE != WINDOW && kk < p.sinks;
    int lo = (int)max(0L, (long)kk - p.right) - at;                  // the window's queries [lo, hi]
    int hi = (int)min((long)len - 1, (long)kk + p.left) - at;
    int first = p.causal ? kk - at : -at, last = len - 1 - at;       // a sink's
    if (kk >= len) hi = lo - 1;
    if (kk >= len || !sink) first = 1, last = 0;
    if (hi < lo) lo = 1 << 29, hi = lo;
    const unsigned w = (unsigned)(hi - lo);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int t = row_of(r);
      const bool window = (unsigned)(t - lo) <= w;
      const bool any = t >= first && t <= last;
      const bool keep = MODE == WINDOW ? window : MODE == SINK ? any && !window : window || any;
      if (!keep) sc[r] = 0.f;
    }
  }

  // Lane column = query qq, elements = the keys k + 4 hh + row_of(r): masked ones become v.
  static __device__ __forceinline__ void mask_keys(f32x16& sc, int k, int qq, int lane, float v, int len,
                                                   const AttnOpArgs& p) {
    const int at = k + 4 * (lane >> 5);
    int lo = qq - p.left - at, hi = (int)min((long)len - 1, (long)qq + p.right) - at;
    int sink = min(p.sinks, p.causal ? min(len, qq + 1) : len) - at;  // keys below it are visible
    if (qq >= len) hi = lo - 1, sink = -1;
    if (hi < lo) lo = 1 << 29, hi = lo;
    const unsigned w = (unsigned)(hi - lo);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int t = row_of(r);
      if (!((unsigned)(t - lo) <= w || t < sink)) sc[r] = v;
    }
  }
  // body(stage, it) for n steps, whose operands issue(stage, it) copies: the next
  // step's while this one computes.  The caller has issued step 0.
  template <class Issue, class Body>
  static __device__ __forceinline__ void pipeline(int n, char* lds, int stage, Issue issue, Body body) {
    stage_sync();
    for (int it = 0; it < n; ++it) {
      if (it + 1 < n) issue(lds + (~it & 1) * stage, it + 1);
      body(lds + (it & 1) * stage, it);
      stage_sync();
    }
  }

  // -- forward -----------------------------------------------------------------
  // Scores and the reference m are in base 2 with a bias, and as the products give
  // them without.  Exponents come from their difference: at a row's only visible
  // token it is zero, so its probability is exactly one, o its value and dS zero.
  // (The rounded product of a score with sl2, less that of m, is not zero.  us of the
  // forward with that and with differences: 32 / 8 heads of 128, s 8192, window 1024:
  // 191, 197; 16 heads of 64, s 16384, window 256: 64, 66.)
  static __device__ __forceinline__ float base2(float x, const AttnOpArgs& p) { return BIAS ? x : x * p.sl2; }
  struct Fwd {
    f32x16 o[NB];
    float m, l;
  };
  static __device__ __forceinline__ void reset(Fwd& st) {
#pragma unroll
    for (int i = 0; i < NB; ++i) zero(st.o[i]);
    st.m = kNone;
    st.l = 0.f;
  }
  // Scores of N blocks of 32 keys from k0 to exponentials, with the state moved to their maximum.
  template <int N>
  static __device__ __forceinline__ void softmax(Fwd& st, f32x16 (&sc)[N], int k0, int q0, int qq, int lane, int len,
                                                 const float* table, const AttnOpArgs& p) {
    if constexpr (BIAS) {
      const int rel = k0 - q0;
      const bool near = wave_uniform(rel + 32 * N - 1 > -p.far && rel - 31 < p.far);
      const int e = k0 + 4 * (lane >> 5) - qq + table_off(p);
      float c = 0.f;
      if (!near) c = rel < 0 ? table[0] : table[table_len(p) - 1];
#pragma unroll
      for (int j = 0; j < N; ++j) add_bias<1>(sc[j], table, e + 32 * j, c, near, p);
    }
    if (wave_uniform(!all_visible<32, 32 * N>(p, q0, k0, len))) {
#pragma unroll
      for (int j = 0; j < N; ++j) mask_keys(sc[j], k0 + 32 * j, qq, lane, -INFINITY, len, p);
    }
    float mx = -INFINITY;
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[j][r]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    // the reference moves when a row's maximum exceeds it by more than 2^8
    const bool grow = base2(mx - st.m, p) > 8.f;
    if (__any(grow)) {
      const float m_new = grow ? mx : st.m;
      const float alpha = __builtin_amdgcn_exp2f(base2(st.m - m_new, p));
      st.m = m_new;
      st.l *= alpha;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) st.o[b][r] *= alpha;
    }
    float ls = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float e = __builtin_amdgcn_exp2f(base2(sc[j][r] - st.m, p));
        sc[j][r] = e;
        ls += e;
      }
    st.l += ls;
  }
  // One block of 64 keys.  D = do.o keeps the rounding of the
  // exponentials to bf16, as the root of the sum of squares of a row's
  // probabilities next to dS's own: it counts where rows see few tokens (rel-L2
  // of dq, 12 tokens a sequence: 2.8e-3, against 2.4e-3), and where the bias
  // gradient sums it over the far bucket, which holds most of a long row
  // (2133 tokens, both directions, 8 buckets: 4.1e-3, against 1.7e-3).  There the
  // forward also adds what the rounding drops (FINE; us, 32 heads of 128, s 2048, with
  // a bias: 65 -> 78).
  template <bool FINE>
  static __device__ __forceinline__ void fwd_tile(Fwd& st, const Rows& qf, const char* kt, const char* vt, const Offs& of,
                                                  int k0, int q0, int qq, int lane, int len, const float* table,
                                                  const AttnOpArgs& p) {
    if (none_visible<64>(p, q0, k0, len)) return;
    f32x16 sc[2];
    zero(sc[0]);
    zero(sc[1]);
    T::score2(sc[0], kt, 0, qf, sc[1], kt, 1, qf, of, lane);
    softmax<2>(st, sc, k0, q0, qq, lane, len, table, p);
    T::template outer<FINE>(st.o, vt, 0, sc[0], of, lane);
    T::template outer<FINE>(st.o, vt, 1, sc[1], of, lane);
  }

  static constexpr int TILE = 2 * T::OWN, STAGE = 2 * TILE;

  template <bool FINE>
  static __device__ __forceinline__ void fwd(const AttnOpArgs& p, char* lds) {
    float* const table = (float*)(lds + 2 * STAGE);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int bh = p.batch * p.heads, nqb = (p.s + 127) / 128;
    const int z = blockIdx.x % bh, qb = nqb - 1 - blockIdx.x / bh;
    const int b = z / p.heads, h = z % p.heads;
    const int len = length(p, b);
    const int q0 = qb * 128 + 32 * wave, qq = q0 + (lane & 31);
    const Steps steps = key_steps<64>(p, qb * 128, qb * 128 + 127, len);
    Src ks, vs;
    ks.set(base(p.k, b, h / p.group), p.k.t, len);
    vs.set(base(p.v, b, h / p.group), p.v.t, len);
    auto issue = [&](char* t, int it) {
      const int k0 = steps.tile(it) * 64;
      T::copy(t, ks, wave, lane, k0, len, p.d);
      T::copy(t + TILE, vs, wave, lane, k0, len, p.d);
    };
    if (steps.n > 0) issue(lds, 0);
    Rows qf;
    T::rows(qf, base(p.q, b, h), p.q.t, qq, len, lane, p.d);
    if constexpr (BIAS) fill_table(p, h, table);
    Offs of;
    of.init(lane);
    Fwd st;
    reset(st);
    pipeline(steps.n, lds, STAGE, issue, [&](char* cur, int it) {
      fwd_tile<FINE>(st, qf, cur, cur + TILE, of, steps.tile(it) * 64, q0, qq, lane, len, table, p);
    });
    fwd_store(st, p, b, h, q0, qq, len, lane, lds + wave * (STAGE / 4));
  }

  // 32 queries a workgroup: its waves take every fourth block of 32 keys, with
  // tiles of their own (or none), and join their sums through LDS.
  static constexpr int SUMS = NB * 4096, OWN = 2 * T::OWN > SUMS ? 2 * T::OWN : SUMS;
  template <bool FINE>
  static __device__ __forceinline__ void fwd32(const AttnOpArgs& p, char* lds) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    char* const own = lds + wave * OWN;
    float2* const stats = (float2*)(lds + 4 * OWN);  // [wave][lane]
    float* const table = (float*)(lds + 4 * OWN + 2048);
    const int bh = p.batch * p.heads, nqb = (p.s + 31) / 32;
    const int z = blockIdx.x % bh, q0 = 32 * (nqb - 1 - blockIdx.x / bh), qq = q0 + (lane & 31);
    const int b = z / p.heads, h = z % p.heads;
    const int len = length(p, b);
    const Steps steps = key_steps<32>(p, q0, q0 + 31, len);
    Src ks, vs;
    ks.set(base(p.k, b, h / p.group), p.k.t, len);
    vs.set(base(p.v, b, h / p.group), p.v.t, len);
    auto issue = [&](int it) {
      const int k0 = steps.tile(it) * 32;
      T::copy_own(own, ks, lane, k0, len, p.d);
      T::copy_own(own + T::OWN, vs, lane, k0, len, p.d);
    };
    if (wave < steps.n) issue(wave);
    Rows qf;
    T::rows(qf, base(p.q, b, h), p.q.t, qq, len, lane, p.d);
    Offs of;
    of.init(lane);
    Fwd st;
    reset(st);
    if constexpr (BIAS) {
      fill_table(p, h, table);
      __syncthreads();
    }
    for (int it = wave; it < steps.n; it += 4) {
      T::own_landed();
      const int k0 = steps.tile(it) * 32;
      if (!none_visible<32>(p, q0, k0, len)) {
        f32x16 sc[1];
        zero(sc[0]);
        T::score1(sc[0], T::block(ks, own, k0, len, p.d), qf, of, lane);
        const Block vb = T::block(vs, own + T::OWN, k0, len, p.d);
        softmax<1>(st, sc, k0, q0, qq, lane, len, table, p);
        T::template outer<FINE>(st.o, vb, 0, sc[0], of, lane);
      }
      T::own_read();
      if (it + 4 < steps.n) issue(it + 4);
    }
    put<NB>(st.o, own, lane);
    stats[wave * 64 + lane] = make_float2(st.m, st.l);
    __syncthreads();
    // every wave joins the four states, wave 0 the statistics, each the columns it stores
    float m = kNone, scale[4];
    float l = 0.f;
#pragma unroll
    for (int u = 0; u < 4; ++u) m = fmaxf(m, stats[u * 64 + lane].x);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float2 t = stats[u * 64 + lane];
      scale[u] = __builtin_amdgcn_exp2f(base2(t.x - m, p));
      l += scale[u] * t.y;
    }
    st.m = m;
    st.l = l;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      zero(st.o[i]);
      if (i % 4 != wave) continue;
#pragma unroll
      for (int u = 0; u < 4; ++u) add_scaled(st.o[i], lds + u * OWN, i, lane, scale[u]);
    }
    float inv;
    const bool some = finish(st, inv, qq, len);
    E* const to = out(p.o, b, h);
    E* const rest = T::REST && p.m ? (E*)p.rest + ((long)b * p.s * p.heads + h) * p.d : nullptr;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      if (i % 4 != wave) continue;
      T::store_cols(st.o[i], to, p.o.t, q0, p.s, i, lane, inv, p.d);
      if constexpr (T::REST) {
        if (!rest) continue;
        T::A::keep_rest(st.o[i], inv);
        T::store_cols(st.o[i], rest, (long)p.heads * p.d, q0, p.s, i, lane, 1.0f, p.d);
      }
    }
    if (p.m && wave == 0) store_stats(st, p, z, qq, some, lane);
  }

  // A wave's blocks to its area, in chunks of 16 bytes a lane; and one of them back, scaled and added.
  template <int N>
  static __device__ __forceinline__ void put(const f32x16 (&a)[N], char* area, int lane) {
    float4* to = (float4*)area + lane;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        to[(4 * i + c) * 64] = make_float4(a[i][4 * c], a[i][4 * c + 1], a[i][4 * c + 2], a[i][4 * c + 3]);
  }
  static __device__ __forceinline__ void add_scaled(f32x16& a, const char* area, int i, int lane, float mul) {
    const float4* from = (const float4*)area + lane;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float4 v = from[(4 * i + c) * 64];
      a[4 * c] += v.x * mul;
      a[4 * c + 1] += v.y * mul;
      a[4 * c + 2] += v.z * mul;
      a[4 * c + 3] += v.w * mul;
    }
  }

  // 1 / sum of this lane's row (0 for a row without a visible token, whose sums become zeros);
  // whether there is one.
  static __device__ __forceinline__ bool finish(Fwd& st, float& inv, int qq, int len) {
    st.l += __shfl_xor(st.l, 32, 64);
    const bool some = st.l > 0.f || st.l != st.l;
    inv = some ? 1.0f / st.l : 0.f;
    if (qq >= len) {
#pragma unroll
      for (int i = 0; i < NB; ++i) zero(st.o[i]);
    }
    return some;
  }
  static __device__ __forceinline__ void store_stats(const Fwd& st, const AttnOpArgs& p, int z, int qq, bool some,
                                                     int lane) {
    if (lane >= 32 || qq >= p.spad) return;
    p.m[(long)z * p.spad + qq] = some ? st.m : 0.f;
    p.l[(long)z * p.spad + qq] = some ? __builtin_amdgcn_logf(st.l) : 0.f;
  }
  static __device__ __forceinline__ void fwd_store(Fwd& st, const AttnOpArgs& p, int b, int h, int q0, int qq, int len,
                                                   int lane, char* area) {
    float inv;
    const bool some = finish(st, inv, qq, len);
    T::store(st.o, area, out(p.o, b, h), p.o.t, q0, p.s, lane, inv, p.d);
    if (!p.m) return;
    if constexpr (T::REST) {
#pragma unroll
      for (int i = 0; i < NB; ++i) T::A::keep_rest(st.o[i], inv);
      T::store(st.o, area, (E*)p.rest + ((long)b * p.s * p.heads + h) * p.d, (long)p.heads * p.d, q0, p.s, lane, 1.0f,
               p.d);
    }
    store_stats(st, p, b * p.heads + h, qq, some, lane);
  }

  // -- dq, dbias and D -----------------------------------------------------------
  // A wave's 32 queries: rows of q and dout, and the statistics.  With a bias
  // what turns do.v into dS / 2^(x - m) = do.v / sum - D / sum: inv, and D times it.
  struct Queries {
    Rows q, d;
    float m, l, inv, D;
  };
  static __device__ __forceinline__ void load_queries(Queries& w, const AttnOpArgs& p, int b, int h, int qq, int len,
                                                      int lane, bool write) {
    const long row = ((long)b * p.heads + h) * p.spad + qq;
    T::rows(w.q, base(p.q, b, h), p.q.t, qq, len, lane, p.d);
    T::rows(w.d, base(p.dout, b, h), p.dout.t, qq, len, lane, p.d);
    f32x16 a;
    zero(a);
    {
      Rows of;
      T::rows(of, base(p.o, b, h), p.o.t, qq, len, lane, p.d);
      T::dot(a, of, w.d);
      if constexpr (T::REST) {
        T::rows(of, (const E*)p.rest + ((long)b * p.s * p.heads + h) * p.d, (long)p.heads * p.d, qq, len, lane, p.d);
        T::dot(a, of, w.d);
      }
    }
    // the diagonal: row lane % 32 of column lane % 32, held by one half of the wave
    const int want = (lane & 31) - 4 * (lane >> 5);
    float D = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (row_of(r) == want) D = a[r];
    D = ((lane >> 2) & 1) == (lane >> 5) ? D : 0.f;
    D += __shfl_xor(D, 32, 64);
    if (write && lane < 32 && qq < p.spad) p.drow[row] = qq < len ? D : 0.f;
    w.m = qq < p.s ? p.m[row] : 0.f;
    w.l = qq < p.s ? p.l[row] : 0.f;
    w.inv = qq < p.s ? __builtin_amdgcn_exp2f(-w.l) : 0.f;
    w.D = BIAS ? D * w.inv : D;
  }

  // Sums of dS by distance: this wave's table of near ones, far ones on either side.
  struct Sums {
    float* near;
    float left, right;
  };
  // A zeroed table for every wave, behind the bias.
  static __device__ __forceinline__ Sums start_sums(const AttnOpArgs& p, float* table, int wave) {
    float* const all = table + table_len(p);
    for (int e = threadIdx.x; e < 4 * table_len(p); e += 256) all[e] = 0.f;
    return {all + wave * table_len(p), 0.f, 0.f};
  }
  // The sums of each bucket over the four tables, in order, by eight lanes each.  After a barrier.
  static __device__ __forceinline__ void finish_sums(const AttnOpArgs& p, Sums& s, float* table, int wave, int lane,
                                                     float* to) {
    const int n = table_len(p), off = table_off(p);
    const float* const all = table + n;
    float* const fars = table;  // the bias is no longer needed
    const float fl = wave_sum(s.left), fr = wave_sum(s.right);
    if (lane == 0) fars[wave] = fl, fars[4 + wave] = fr;
    __syncthreads();
    const int side = p.causal ? p.buckets : p.buckets / 2, part = threadIdx.x % 8;
    for (int c0 = 0; c0 < p.buckets; c0 += 32) {
      const int c = min(c0 + (int)threadIdx.x / 8, p.buckets - 1);
      const bool ahead = c >= side;
      const int cs = ahead ? c - side : c;
      // its distances [n0, n1); distance 0 counts once
      const int n0 = max((int)p.first[cs], ahead ? 1 : 0);
      const int n1 = cs == side - 1 ? (ahead ? n - off : off + 1) : p.first[cs + 1];
      float t = 0.f;
      for (int e = n0 + part; e < n1; e += 8) {
        const float* x = all + (ahead ? off + e : off - e);
#pragma unroll
        for (int i = 0; i < 4; ++i) t += x[i * n];
      }
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) t += __shfl_xor(t, o, 64);
      if (cs == side - 1) {
        const float* f = fars + (ahead ? 4 : 0);
        t += f[0] + f[1] + f[2] + f[3];
      }
      if (part == 0 && c0 + (int)threadIdx.x / 8 < p.buckets) to[c] = t;
    }
  }

  // acc += dS times the 32 keys from k (rows j of the tiles).  FINE (rows of few
  // tokens): with what the rounding of dS drops, which there costs little and is not
  // averaged over a row.
  template <bool FINE>
  static __device__ __forceinline__ void dq_block(f32x16 (&acc)[NB], const Queries& w, const Block& kt, const Block& vt,
                                                  int j, const Offs& of, int k, int q0, int qq, int lane, int len,
                                                  const float* table, Sums& sums, const AttnOpArgs& p) {
    if (none_visible<32>(p, q0, k, len)) return;
    f32x16 sc, dp;
    zero(sc);
    zero(dp);
    T::score2(sc, kt, j, w.q, dp, vt, j, w.d, of, lane);
    const int rel = k - q0;
    const bool near = BIAS && wave_uniform(rel + 31 > -p.far && rel - 31 < p.far);
    const int e = k + 4 * (lane >> 5) - qq + (BIAS ? table_off(p) : 0);
    if constexpr (BIAS) {
      float c = 0.f;
      if (!near) c = rel < 0 ? table[0] : table[table_len(p) - 1];
      add_bias<1>(sc, table, e, c, near, p);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = __builtin_amdgcn_exp2f(BIAS ? sc[r] - w.m : fmaf(sc[r] - w.m, p.sl2, -w.l));
    if (wave_uniform(!all_visible<32, 32>(p, q0, k, len))) mask_keys(sc, k, qq, lane, 0.f, len, p);
#pragma unroll
    for (int r = 0; r < 16; ++r) dp[r] = sc[r] * (BIAS ? fmaf(dp[r], w.inv, -w.D) : dp[r] - w.D);
    if constexpr (BIAS) {
      if (near) {
        add_diagonals(sums.near + e, dp, lane);
      } else {
        float t = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) t += dp[r];
        if (rel < 0)
          sums.left += t;
        else
          sums.right += t;
      }
    }
    T::template outer<FINE>(acc, kt, j, dp, of, lane);
  }

  template <bool FINE>
  static __device__ __forceinline__ void dq(const AttnOpArgs& p, char* lds) {
    float* const table = (float*)(lds + 2 * STAGE);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int bh = p.batch * p.heads, nqb = (p.s + 127) / 128;
    const int z = blockIdx.x % bh, qb = nqb - 1 - blockIdx.x / bh;
    const int b = z / p.heads, h = z % p.heads;
    const int len = length(p, b);
    const int q0 = qb * 128 + 32 * wave, qq = q0 + (lane & 31);
    const Steps steps = key_steps<64>(p, qb * 128, qb * 128 + 127, len);
    Src ks, vs;
    ks.set(base(p.k, b, h / p.group), p.k.t, len);
    vs.set(base(p.v, b, h / p.group), p.v.t, len);
    auto issue = [&](char* t, int it) {
      const int k0 = steps.tile(it) * 64;
      T::copy(t, ks, wave, lane, k0, len, p.d);
      T::copy(t + TILE, vs, wave, lane, k0, len, p.d);
    };
    if (steps.n > 0) issue(lds, 0);
    Queries w;
    load_queries(w, p, b, h, qq, len, lane, true);
    Sums sums = {nullptr, 0.f, 0.f};
    if constexpr (BIAS) {
      fill_table(p, h, table);
      sums = start_sums(p, table, wave);
    }
    Offs of;
    of.init(lane);
    f32x16 acc[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) zero(acc[i]);
    pipeline(steps.n, lds, STAGE, issue, [&](char* cur, int it) {
      const int k0 = steps.tile(it) * 64;
#pragma unroll 1
      for (int j = 0; j < 2; ++j)
        dq_block<FINE>(acc, w, cur, cur + TILE, j, of, k0 + 32 * j, q0, qq, lane, len, table, sums, p);
    });
    if (qq >= len) {
#pragma unroll
      for (int i = 0; i < NB; ++i) zero(acc[i]);
    }
    T::store(acc, lds + wave * (STAGE / 4), out(p.dq, b, h), p.dq.t, q0, p.s, lane, p.scale, p.d);
    if constexpr (BIAS) finish_sums(p, sums, table, wave, lane, p.bpart + ((long)z * nqb + qb) * p.buckets);
  }

  // 32 queries a workgroup, as fwd32.
  template <bool FINE>
  static __device__ __forceinline__ void dq32(const AttnOpArgs& p, char* lds) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    char* const own = lds + wave * OWN;
    float* const table = (float*)(lds + 4 * OWN);
    const int bh = p.batch * p.heads, nqb = (p.s + 31) / 32;
    const int z = blockIdx.x % bh, qb = nqb - 1 - blockIdx.x / bh, q0 = 32 * qb, qq = q0 + (lane & 31);
    const int b = z / p.heads, h = z % p.heads;
    const int len = length(p, b);
    const Steps steps = key_steps<32>(p, q0, q0 + 31, len);
    Src ks, vs;
    ks.set(base(p.k, b, h / p.group), p.k.t, len);
    vs.set(base(p.v, b, h / p.group), p.v.t, len);
    auto issue = [&](int it) {
      const int k0 = steps.tile(it) * 32;
      T::copy_own(own, ks, lane, k0, len, p.d);
      T::copy_own(own + T::OWN, vs, lane, k0, len, p.d);
    };
    if (wave < steps.n) issue(wave);
    Queries w;
    load_queries(w, p, b, h, qq, len, lane, wave == 0);
    Sums sums = {nullptr, 0.f, 0.f};
    Offs of;
    of.init(lane);
    f32x16 acc[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) zero(acc[i]);
    if constexpr (BIAS) {
      fill_table(p, h, table);
      sums = start_sums(p, table, wave);
      __syncthreads();
    }
    for (int it = wave; it < steps.n; it += 4) {
      T::own_landed();
      const int k0 = steps.tile(it) * 32;
      dq_block<FINE>(acc, w, T::block(ks, own, k0, len, p.d), T::block(vs, own + T::OWN, k0, len, p.d), 0, of, k0, q0, qq,
                     lane, len, table, sums, p);
      T::own_read();
      if (it + 4 < steps.n) issue(it + 4);
    }
    put<NB>(acc, own, lane);
    __syncthreads();
    E* const to = out(p.dq, b, h);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      if (i % 4 != wave) continue;
      zero(acc[i]);
      if (qq < len) {
#pragma unroll
        for (int u = 0; u < 4; ++u) add_scaled(acc[i], lds + u * OWN, i, lane, 1.0f);
      }
      T::store_cols(acc[i], to, p.dq.t, q0, p.s, i, lane, p.scale, p.d);
    }
    if constexpr (BIAS) finish_sums(p, sums, table, wave, lane, p.bpart + ((long)z * nqb + qb) * p.buckets);
  }

  // -- dk and dv -------------------------------------------------------------------
  static __device__ __forceinline__ void load_rows16(f32x16& row, const float* from) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float4 v = *(const float4*)__builtin_assume_aligned(from + 8 * c, 16);
      row[4 * c] = v.x;
      row[4 * c + 1] = v.y;
      row[4 * c + 2] = v.z;
      row[4 * c + 3] = v.w;
    }
  }
  // dk, dv += the 32 queries from q (rows j of the tiles), with their statistics.
  template <int MODE, bool FINE>
  static __device__ __forceinline__ void dkv_block(f32x16 (&dk)[NB], f32x16 (&dv)[NB], const Rows& kf, const Rows& vf,
                                                   const Block& qt, const Block& dt, int j, const float* m, const float* l,
                                                   const float* D, const Offs& of, int q, int k0, int kk, int lane,
                                                   int len, const float* table, const AttnOpArgs& p) {
    if (none_of<MODE>(p, q, k0, len)) return;
    f32x16 sc, dp;
    zero(sc);
    zero(dp);
    T::score2(sc, qt, j, kf, dp, dt, j, vf, of, lane);
    if constexpr (BIAS) {
      const int rel = k0 - q;
      const bool near = wave_uniform(rel + 31 > -p.far && rel - 31 < p.far);
      float c = 0.f;
      if (!near) c = rel < 0 ? table[0] : table[table_len(p) - 1];
      add_bias<-1>(sc, table, kk - q - 4 * (lane >> 5) + table_off(p), c, near, p);
    }
    const int at = 4 * (lane >> 5);
    f32x16 row;  // a statistic of the block's queries
    load_rows16(row, m + at);
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] -= row[r];
    load_rows16(row, l + at);
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = __builtin_amdgcn_exp2f(BIAS ? sc[r] - row[r] : fmaf(sc[r], p.sl2, -row[r]));
    load_rows16(row, D + at);
    if (wave_uniform(!all_of<MODE>(p, q, k0, len))) mask_queries<MODE>(sc, q, kk, lane, len, p);
#pragma unroll
    for (int r = 0; r < 16; ++r) dp[r] = sc[r] * (dp[r] - row[r]);
    T::template outer<FINE>(dv, dt, j, sc, of, lane);
    T::template outer<FINE>(dk, qt, j, dp, of, lane);
  }

  // This wave's rows k0.. of dk or dv as share `n` of the sinks' rows, or as the
  // share of a part of the heads.
  static __device__ __forceinline__ float* share(const AttnOpArgs& p, int z, int n, int which, int k0) {
    return p.spart + ((((long)z * (1 + p.chunks * p.parts) + n) * 2 + which) * p.sink_rows + k0) * HD;
  }
  static __device__ __forceinline__ float* part_share(const AttnOpArgs& p, int z, int part, int which, int k0) {
    return p.gpart + ((((long)z * p.parts + part) * 2 + which) * p.part_rows + k0) * HD;
  }
  // The heads [first, second) of a part.
  static __device__ __forceinline__ int2 heads_of(const AttnOpArgs& p, int hk, int part) {
    return make_int2(hk * p.group + part * p.group / p.parts, hk * p.group + (part + 1) * p.group / p.parts);
  }
  static __device__ __forceinline__ void store_share(const f32x16& a, float* to, int i, int lane) {
    to += (lane & 31) * HD + 32 * i + 4 * (lane >> 5);
#pragma unroll
    for (int c = 0; c < 4; ++c)
      *(float4*)(to + 8 * c) = make_float4(a[4 * c], a[4 * c + 1], a[4 * c + 2], a[4 * c + 3]);
  }

  // A stage: a Q tile, a dO tile and the row vectors m, l, D of 64 queries.
  static constexpr int KSTAGE = 2 * TILE + 3 * 1024;

  // dbias[h, c] = sum of the query blocks' shares in the order of (sequence,
  // block): 256 / buckets groups of threads take every g-th share, then add up.
  // By workgroups behind the others of the dk and dv kernels, which run after
  // the one that leaves the shares.
  static __device__ __forceinline__ void dbias(const AttnOpArgs& p, int h, float* red) {
    const int groups = 256 / p.buckets, g = threadIdx.x / p.buckets, c = threadIdx.x % p.buckets;
    const int n = p.batch * p.bias_blocks;
    float t = 0.f;
    if (g < groups)
#pragma unroll 4
      for (int i = g; i < n; i += groups)
        t += p.bpart[(((long)(i / p.bias_blocks) * p.heads + h) * p.bias_blocks + i % p.bias_blocks) * p.buckets + c];
    red[threadIdx.x] = t;
    __syncthreads();
    if (g != 0) return;
    for (int k = 1; k < groups; ++k) t += red[k * p.buckets + c];
    const long at = (long)h * p.buckets + c;
    if (p.bias_f32)
      ((float*)p.dbias)[at] = t;
    else
      ((bf16*)p.dbias)[at] = (bf16)t;
  }

  template <bool FINE>
  static __device__ __forceinline__ void dkv(const AttnOpArgs& p, char* lds) {
    const int bk = p.batch * p.kv_heads, z = blockIdx.x % bk, kb = blockIdx.x / bk;
    const int nkb = (p.s + 127) / 128 * p.parts, units = nkb + p.sink_rows / 32 * p.chunks * p.parts;
    if constexpr (BIAS)
      if (kb >= units) return dbias(p, blockIdx.x - units * bk, (float*)lds);
    if (kb >= nkb) return dkv_sinks<FINE>(p, lds, z, kb - nkb);
    const int part = kb % p.parts;
    float* const table = (float*)(lds + 2 * KSTAGE);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = z / p.kv_heads, hk = z % p.kv_heads;
    const int len = length(p, b);
    const int2 heads = heads_of(p, hk, part);
    const int K0 = kb / p.parts * 128, k0 = K0 + 32 * wave, kk = k0 + (lane & 31);
    // the queries whose windows hold these keys
    const int qlo = (int)max(0L, (long)K0 - p.right);
    const int qhi = K0 < len ? (int)min((long)len - 1, (long)K0 + 127 + p.left) : -1;
    const int t0 = qlo / 64, nt = qhi >= qlo ? qhi / 64 - t0 + 1 : 0;
    Src qs, ds;
    // step i: tile i % nt of head i / nt of the group; steps are issued and
    // computed in order, so both count along
    int gi = 0, ti = 0, gc = 0, tc = 0;
    auto issue = [&](char* t, int) {
      const int h = heads.x + gi, row0 = (t0 + ti) * 64;
      if (ti == 0) {
        qs.set(base(p.q, b, h), p.q.t, len);
        ds.set(base(p.dout, b, h), p.dout.t, len);
      }
      T::copy(t, qs, wave, lane, row0, len, p.d);
      T::copy(t + TILE, ds, wave, lane, row0, len, p.d);
      if (wave < 3)
        T::vec(t + 2 * TILE + 1024 * wave,
               (wave == 0 ? p.m : wave == 1 ? p.l : p.drow) + ((long)b * p.heads + h) * p.spad + row0, lane);
      if (++ti == nt) ti = 0, ++gi;
    };
    if (nt > 0) issue(lds, 0);
    Rows kf, vf;
    T::rows(kf, base(p.k, b, hk), p.k.t, kk, len, lane, p.d);
    T::rows(vf, base(p.v, b, hk), p.v.t, kk, len, lane, p.d);
    Offs of;
    of.init(lane);
    f32x16 dk[NB], dv[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      zero(dk[i]);
      zero(dv[i]);
    }
    pipeline(nt * (heads.y - heads.x), lds, KSTAGE, issue, [&](char* cur, int) {
      if constexpr (BIAS) {
        if (tc == 0) {  // the first tile of a head: its bias
          fill_table(p, heads.x + gc, table);
          __syncthreads();
        }
      }
      const float* vec = (const float*)(cur + 2 * TILE);
#pragma unroll 1
      for (int j = 0; j < 2; ++j)
        dkv_block<WINDOW, FINE>(dk, dv, kf, vf, cur, cur + TILE, j, vec + 32 * j, vec + 256 + 32 * j, vec + 512 + 32 * j, of,
                          (t0 + tc) * 64 + 32 * j, k0, kk, lane, len, table, p);
      if (++tc == nt) tc = 0, ++gc;
    });
    if (kk >= len) {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        zero(dk[i]);
        zero(dv[i]);
      }
    }
    if (p.parts > 1 || (p.chunks && k0 < p.sink_rows)) {
      float* const to_k = p.parts > 1 ? part_share(p, z, part, 0, k0) : share(p, z, 0, 0, k0);
      float* const to_v = p.parts > 1 ? part_share(p, z, part, 1, k0) : share(p, z, 0, 1, k0);
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        store_share(dk[i], to_k, i, lane);
        store_share(dv[i], to_v, i, lane);
      }
      return;
    }
    char* const area = lds + wave * (STAGE / 4);
    T::store(dk, area, out(p.dk, b, hk), p.dk.t, k0, p.s, lane, p.scale, p.d);
    T::store(dv, area, out(p.dv, b, hk), p.dv.t, k0, p.s, lane, 1.0f, p.d);
  }

  // 32 keys a workgroup: its waves take every fourth block of 32 queries, of
  // every head of the group, with tiles of their own.  MODE SINK: the sinks among
  // the keys, for the queries of a chunk that see them as such.
  static constexpr int KOWN = OWN + (T::DIRECT ? 0 : 3 * 1024);
  template <int MODE, bool FINE>
  static __device__ __forceinline__ void dkv32(const AttnOpArgs& p, char* lds, int z, int k0, int chunk, int part) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    char* const own = lds + wave * KOWN;
    float* const table = (float*)(lds + 4 * KOWN);
    const int b = z / p.kv_heads, hk = z % p.kv_heads;
    const int len = length(p, b);
    const int kk = k0 + (lane & 31);
    int qlo, qhi;
    if (MODE == SINK) {
      qlo = max(p.causal ? (int)min((long)p.s, (long)k0 + p.left + 1) : 0, chunk * p.chunk_len);
      qhi = (int)min((long)len, (chunk + 1L) * p.chunk_len) - 1;
    } else if (MODE == BOTH && k0 < p.sinks) {
      qlo = p.causal ? k0 : 0;
      qhi = len - 1;
    } else {
      qlo = (int)max(0L, (long)k0 - p.right);
      qhi = (int)min((long)len - 1, (long)k0 + 31 + p.left);
    }
    if (k0 >= len) qhi = -1;
    const int t0 = qlo / 32, nt = qhi >= qlo ? qhi / 32 - t0 + 1 : 0;
    Rows kf, vf;
    T::rows(kf, base(p.k, b, hk), p.k.t, kk, len, lane, p.d);
    T::rows(vf, base(p.v, b, hk), p.v.t, kk, len, lane, p.d);
    Offs of;
    of.init(lane);
    f32x16 dk[NB], dv[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      zero(dk[i]);
      zero(dv[i]);
    }
    const int2 heads = heads_of(p, hk, part);
    for (int h = heads.x; h < heads.y; ++h) {
      Src qs, ds;
      qs.set(base(p.q, b, h), p.q.t, len);
      ds.set(base(p.dout, b, h), p.dout.t, len);
      const long rows = ((long)b * p.heads + h) * p.spad;
      auto issue = [&](int it) {
        const int row0 = (t0 + it) * 32;
        T::copy_own(own, qs, lane, row0, len, p.d);
        T::copy_own(own + T::OWN, ds, lane, row0, len, p.d);
        T::vec(own + OWN, p.m + rows + row0, lane, 32);
        T::vec(own + OWN + 1024, p.l + rows + row0, lane, 32);
        T::vec(own + OWN + 2048, p.drow + rows + row0, lane, 32);
      };
      if (wave < nt) issue(wave);
      if constexpr (BIAS) {
        __syncthreads();  // every wave is done with the last head's bias
        fill_table(p, h, table);
        __syncthreads();
      }
      for (int it = wave; it < nt; it += 4) {
        T::own_landed();
        const int row0 = (t0 + it) * 32;
        dkv_block<MODE, FINE>(dk, dv, kf, vf, T::block(qs, own, row0, len, p.d), T::block(ds, own + T::OWN, row0, len, p.d),
                              0, T::vec_of(own + OWN, p.m + rows + row0), T::vec_of(own + OWN + 1024, p.l + rows + row0),
                              T::vec_of(own + OWN + 2048, p.drow + rows + row0), of, row0, k0, kk, lane, len, table, p);
        T::own_read();
        if (it + 4 < nt) issue(it + 4);
      }
    }
    // one of the two sums after the other through LDS
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
      if (which)
        put<NB>(dv, own, lane);
      else
        put<NB>(dk, own, lane);
      __syncthreads();
      const AttnOpView& view = which ? p.dv : p.dk;
      const int n = MODE == SINK ? 1 + chunk * p.parts + part : 0;
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        if (i % 4 != wave) continue;
        f32x16 a;
        zero(a);
        if (kk < len) {
#pragma unroll
          for (int u = 0; u < 4; ++u) add_scaled(a, lds + u * KOWN, i, lane, 1.0f);
        }
        if (MODE != SINK && p.parts > 1)
          store_share(a, part_share(p, z, part, which, k0), i, lane);
        else if (p.chunks && k0 < p.sink_rows)
          store_share(a, share(p, z, n, which, k0), i, lane);
        else
          T::store_cols(a, out(view, b, hk), view.t, k0, p.s, i, lane, which ? 1.0f : p.scale, p.d);
      }
    }
  }
  // Unit u of the sinks' workgroups: 32 keys, a chunk of queries, a part of the heads.
  template <bool FINE>
  static __device__ __forceinline__ void dkv_sinks(const AttnOpArgs& p, char* lds, int z, int u) {
    const int n = p.chunks * p.parts;
    dkv32<SINK, FINE>(p, lds, z, u / n * 32, u % n / p.parts, u % p.parts);
  }
  template <bool FINE>
  static __device__ __forceinline__ void dkv_split(const AttnOpArgs& p, char* lds) {
    const int bk = p.batch * p.kv_heads, z = blockIdx.x % bk, kb = blockIdx.x / bk;
    const int nkb = (p.s + 31) / 32 * p.parts, units = nkb + p.sink_rows / 32 * p.chunks * p.parts;
    if constexpr (BIAS)
      if (kb >= units) return dbias(p, blockIdx.x - units * bk, (float*)lds);
    if (kb >= nkb)
      dkv_sinks<FINE>(p, lds, z, kb - nkb);
    else if (p.chunks)
      dkv32<WINDOW, FINE>(p, lds, z, kb / p.parts * 32, 0, kb % p.parts);
    else
      dkv32<BOTH, FINE>(p, lds, z, kb / p.parts * 32, 0, kb % p.parts);
  }

  // LDS of the kernels.
  static size_t table_bytes(const AttnOpArgs& a) { return BIAS ? 4 * (size_t)table_len(a) : 0; }
  static size_t fwd_lds(const AttnOpArgs& a, bool split) {
    return (split ? 4 * OWN + 2048 : 2 * STAGE) + table_bytes(a);
  }
  static size_t dq_lds(const AttnOpArgs& a, bool split) { return (split ? 4 * OWN : 2 * STAGE) + 5 * table_bytes(a); }
  static size_t dkv_lds(const AttnOpArgs& a, bool split) {
    const size_t both = 4 * KOWN, whole = 2 * KSTAGE;
    return (split ? both : a.chunks && both > whole ? both : whole) + table_bytes(a);
  }
};

// Rows of dk and dv from their shares, in order: all rows where the heads are taken
// in parts, the sinks' otherwise.  One workgroup per sequence, key head and 8
// keys; a thread sums 4 columns.
template <class T>
__global__ __launch_bounds__(256) void attn_op_sum_k(AttnOpArgs p) {
  constexpr int HD = T::HD, C4 = HD / 4;
  using E = typename T::E;
  const int bk = p.batch * p.kv_heads, z = blockIdx.x % bk, r8 = blockIdx.x / bk;
  const int b = z / p.kv_heads, h = z % p.kv_heads;
  for (int i = threadIdx.x; i < 8 * 2 * C4; i += 256) {
    const int c = 4 * (i % C4), which = i / C4 % 2, row = 8 * r8 + i / (2 * C4);
    if (row >= p.s || c >= p.d) continue;
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](const float* src, int n, long step) {
#pragma unroll 8
      for (int k = 0; k < n; ++k) {
        const float4 v = *(const float4*)(src + k * step);
        t.x += v.x;
        t.y += v.y;
        t.z += v.z;
        t.w += v.w;
      }
    };
    if (p.parts > 1)
      add(p.gpart + (((long)z * p.parts * 2 + which) * p.part_rows + row) * HD + c, p.parts, 2L * p.part_rows * HD);
    if (p.chunks && row < p.sink_rows) {
      const int first = p.parts > 1 ? 1 : 0, all = 1 + p.chunks * p.parts;
      add(p.spart + ((((long)z * all + first) * 2 + which) * p.sink_rows + row) * HD + c, all - first,
          2L * p.sink_rows * HD);
    }
    const float mul = which ? 1.0f : p.scale;
    const AttnOpView& v = which ? p.dv : p.dk;
    E* o = (E*)v.p + (long)b * v.b + (long)row * v.t + (long)h * v.h + c;
    const E w[4] = {(E)(t.x * mul), (E)(t.y * mul), (E)(t.z * mul), (E)(t.w * mul)};
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = w[e];
  }
}

extern __shared__ __attribute__((aligned(1024))) char attn_op_lds[];

template <class T, bool BIAS, bool FINE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(T::WAVES, T::WAVES))) void attn_op_fwd_k(
    AttnOpArgs p) {
  AttnOp<T, BIAS>::template fwd<FINE>(p, attn_op_lds);
}
template <class T, bool BIAS, bool FINE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(T::FWAVES))) void attn_op_fwd32_k(AttnOpArgs p) {
  AttnOp<T, BIAS>::template fwd32<FINE>(p, attn_op_lds);
}
template <class T, bool BIAS, bool FINE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(T::WAVES, T::WAVES))) void attn_op_dq_k(
    AttnOpArgs p) {
  AttnOp<T, BIAS>::template dq<FINE>(p, attn_op_lds);
}
template <class T, bool BIAS, bool FINE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(T::QWAVES))) void attn_op_dq32_k(AttnOpArgs p) {
  AttnOp<T, BIAS>::template dq32<FINE>(p, attn_op_lds);
}
template <class T, bool BIAS, bool FINE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(T::KWAVES, T::KWAVES))) void attn_op_dkv_k(AttnOpArgs p) {
  AttnOp<T, BIAS>::template dkv<FINE>(p, attn_op_lds);
}
template <class T, bool BIAS, bool FINE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(T::DWAVES))) void attn_op_dkv32_k(AttnOpArgs p) {
  AttnOp<T, BIAS>::template dkv_split<FINE>(p, attn_op_lds);
}

constexpr size_t kLds = 160 * 1024;  // of a compute unit
// Rows of so few tokens, by the masks (sequences' lengths are on the device), take
// the FINE kernels (rel-L2 of dq over that of its own rounding, 142 tokens: 1.50 with
// the coarse forward, 1.46 with the fine one; 4 tokens: 1.4 to 1.9 with the coarse
// backward, 1.0 with the fine one; us of dq and of dk and dv, coarse and fine: 4096
// tokens, 32 heads of 128, window 4: 49, 51 and 62, 68; window 64: 50, 53 and 65, 73).
constexpr int kSeenForward = 160, kSeenBackward = 64;
constexpr size_t kTableMost = 4 * (2 * ATTN_OP_MAX_FAR + 192);

template <class T, bool BIAS, bool FINE>
hipError_t attn_op_fwd_launch(const AttnOpArgs& a, hipStream_t st) {
  using K = AttnOp<T, BIAS>;
  static_assert(4 * K::OWN + 5 * kTableMost <= kLds && 2 * K::STAGE + 5 * kTableMost <= kLds &&
                    4 * K::KOWN + kTableMost <= kLds && 2 * K::KSTAGE + kTableMost <= kLds,
                "LDS at the largest table");
  const bool split = T::DIRECT || a.split_f;
  const long rows = split ? 32 : 128;
  const dim3 grid((unsigned)((a.s + rows - 1) / rows * a.batch * a.heads));
  if (split)
    hipLaunchKernelGGL((attn_op_fwd32_k<T, BIAS, FINE>), grid, dim3(256), K::fwd_lds(a, true), st, a);
  else if constexpr (!T::DIRECT)
    hipLaunchKernelGGL((attn_op_fwd_k<T, BIAS, FINE>), grid, dim3(256), K::fwd_lds(a, false), st, a);
  return hipGetLastError();
}

template <class T, bool BIAS, bool FINE>
hipError_t attn_op_bwd_grids(const AttnOpArgs& a, bool sq, dim3 gq, bool sk, dim3 gk, hipStream_t st) {
  using K = AttnOp<T, BIAS>;
  if (sq)
    hipLaunchKernelGGL((attn_op_dq32_k<T, BIAS, FINE>), gq, dim3(256), K::dq_lds(a, true), st, a);
  else if constexpr (!T::DIRECT)
    hipLaunchKernelGGL((attn_op_dq_k<T, BIAS, FINE>), gq, dim3(256), K::dq_lds(a, false), st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (sk)
    hipLaunchKernelGGL((attn_op_dkv32_k<T, BIAS, FINE>), gk, dim3(256), K::dkv_lds(a, true), st, a);
  else if constexpr (!T::DIRECT)
    hipLaunchKernelGGL((attn_op_dkv_k<T, BIAS, FINE>), gk, dim3(256), K::dkv_lds(a, false), st, a);
  return hipGetLastError();
}

template <class T, bool BIAS>
hipError_t attn_op_bwd_launch(const AttnOpArgs& args, hipStream_t st) {
  AttnOpArgs a = args;
  const bool sq = T::DIRECT || a.split_q, sk = T::DIRECT || a.split_k;
  const long nq = (a.s + (sq ? 31 : 127)) / (sq ? 32 : 128), nk = (a.s + (sk ? 31 : 127)) / (sk ? 32 : 128);
  const dim3 gq((unsigned)(nq * a.batch * a.heads));
  const dim3 gk(
      (unsigned)((nk + (long)a.sink_rows / 32 * a.chunks) * a.parts * a.batch * a.kv_heads + (BIAS ? a.heads : 0)));
  a.bias_blocks = (int)nq;
  hipError_t e;
  if (T::REST && a.seen <= kSeenBackward)
    e = attn_op_bwd_grids<T, BIAS, T::REST>(a, sq, gq, sk, gk, st);
  else
    e = attn_op_bwd_grids<T, BIAS, false>(a, sq, gq, sk, gk, st);
  if (e != hipSuccess || (!a.chunks && a.parts == 1)) return e;
  const long rows = a.parts > 1 || a.sink_rows > a.s ? a.s : a.sink_rows;
  hipLaunchKernelGGL((attn_op_sum_k<T>), dim3((unsigned)((rows + 7) / 8 * a.batch * a.kv_heads)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

#define ATTN_OP_DEFINE(NAME, T)                                                                    \
  hipError_t attn_op_fwd_##NAME(const AttnOpArgs& a, hipStream_t st) {                             \
    return a.bias                   ? attn_op_fwd_launch<T, true, T::REST>(a, st)                  \
           : a.seen <= kSeenForward ? attn_op_fwd_launch<T, false, T::REST>(a, st)                 \
                                    : attn_op_fwd_launch<T, false, false>(a, st);                  \
  }                                                                                                \
  hipError_t attn_op_bwd_##NAME(const AttnOpArgs& a, hipStream_t st) {                             \
    return a.bias ? attn_op_bwd_launch<T, true>(a, st) : attn_op_bwd_launch<T, false>(a, st);      \
  }
