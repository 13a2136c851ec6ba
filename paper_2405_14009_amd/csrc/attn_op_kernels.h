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
// block to a table of its own by distance (the halves of a wave to one
// table each: no two lanes of an instruction meet, every sum has a fixed
// order); far blocks add up in registers.  The tables are summed by buckets
// when the workgroup ends, and over workgroups by a kernel of its own.
//
// D is formed by the same chain of matrix instructions as do.v: where a row
// sees one token only, dS is exactly zero.
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
  static constexpr bool ASYNC = true, REST = true;
  static constexpr int WAVES = 2;  // a SIMD, of the kernels over queries
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
  // 64 floats into a 1 KB area; issued by one wave
  static __device__ __forceinline__ void vec(char* dst, const float* src, int lane) {
    A::load_vec64(make_rsrc(src, 256), dst, lane, 0, 64);
  }
  static __device__ __forceinline__ void rows(Rows& f, const E* base, long ld, int row, int nrows, int lane, int d) {
    A::load_stationary(f, base, ld, row, nrows, lane, d);
  }
  // a0 += block b0 of tile t0 times s0, a1 += block b1 of tile t1 times s1
  static __device__ __forceinline__ void score2(f32x16& a0, const char* t0, int b0, const Rows& s0, f32x16& a1,
                                                const char* t1, int b1, const Rows& s1, const Offs& o, int) {
    A::template two_chains<2>(a0, t0, b0, s0, a1, t1, b1, s1, o.ro);
  }
  // a += rows x times rows y, both from registers
  static __device__ __forceinline__ void dot(f32x16& a, const Rows& x, const Rows& y) {
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks) a = A::mfma(x[ks], y[ks], a);
  }
  // acc += (32 rows j of the tile)^T times the block p
  static __device__ __forceinline__ void outer(f32x16 (&acc)[HD / 32], const char* tile, int j, const f32x16& p,
                                               const Offs& o, int) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const bf16x8 pf = A::pack_half(p, hf);
#pragma unroll
      for (int b = 0; b < HD / 32; ++b) acc[b] = A::mfma(A::rd_tr(tile, o.to, b, 2 * j + hf), pf, acc[b]);
    }
  }
  static __device__ __forceinline__ void store(const f32x16 (&acc)[HD / 32], char* t, E* base, long ld, int row0,
                                               int nrows, int lane, float mul, int d) {
    A::store_rows_lds(acc, t, base, ld, row0, nrows, lane, mul, d);
  }
};

template <int HD_>
struct TileF32 {
  using E = float;
  static constexpr int HD = HD_, LD = HD + 8, TILE = 64 * LD * 4;
  static constexpr bool ASYNC = false, REST = false;
  static constexpr int WAVES = HD > 64 ? 1 : 2;
  // the halves of a wave hold half of the columns each
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
  static __device__ __forceinline__ void copy(char* tile, const Src& s, int wave, int lane, int row0, int nrows, int d) {
    for (int i = wave * 64 + lane; i < 64 * (HD / 4); i += 256) {
      const int r = i / (HD / 4), c = 4 * (i % (HD / 4));
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (row0 + r < nrows && c < d) v = *(const float4*)(s.p + (long)(row0 + r) * s.ld + c);
      *(float4*)((float*)tile + r * LD + c) = v;
    }
  }
  static __device__ __forceinline__ void vec(char* dst, const float* src, int lane) { ((float*)dst)[lane] = src[lane]; }
  static __device__ __forceinline__ void rows(Rows& f, const E* base, long ld, int row, int nrows, int lane, int d) {
#pragma unroll
    for (int k = 0; k < HD / 2; k += 4) {
      const int c = (lane >> 5) * (HD / 2) + k;
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
  static __device__ __forceinline__ void score2(f32x16& a0, const char* t0, int b0, const Rows& s0, f32x16& a1,
                                                const char* t1, int b1, const Rows& s1, const Offs&, int lane) {
    const float* x = (const float*)t0 + (32 * b0 + (lane & 31)) * LD + (lane >> 5) * (HD / 2);
    const float* y = (const float*)t1 + (32 * b1 + (lane & 31)) * LD + (lane >> 5) * (HD / 2);
#pragma unroll
    for (int k = 0; k < HD / 2; k += 4) {
      const float4 u = *(const float4*)(x + k), w = *(const float4*)(y + k);
      a0 = mfma(u.x, s0[k], a0);
      a1 = mfma(w.x, s1[k], a1);
      a0 = mfma(u.y, s0[k + 1], a0);
      a1 = mfma(w.y, s1[k + 1], a1);
      a0 = mfma(u.z, s0[k + 2], a0);
      a1 = mfma(w.z, s1[k + 2], a1);
      a0 = mfma(u.w, s0[k + 3], a0);
      a1 = mfma(w.w, s1[k + 3], a1);
    }
  }
  static __device__ __forceinline__ void dot(f32x16& a, const Rows& x, const Rows& y) {
#pragma unroll
    for (int k = 0; k < HD / 2; ++k) a = mfma(x[k], y[k], a);
  }
  static __device__ __forceinline__ void outer(f32x16 (&acc)[HD / 32], const char* tile, int j, const f32x16& p,
                                               const Offs&, int lane) {
    const float* x = (const float*)tile + (32 * j + 4 * (lane >> 5)) * LD + (lane & 31);
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int b = 0; b < HD / 32; ++b) acc[b] = mfma(x[row_of(r) * LD + 32 * b], p[r], acc[b]);
  }
  static __device__ __forceinline__ void store(const f32x16 (&acc)[HD / 32], char*, E* base, long ld, int row0,
                                               int nrows, int lane, float mul, int d) {
    const int row = row0 + (lane & 31);
    if (row >= nrows) return;
    E* p = base + (long)row * ld + 4 * (lane >> 5);
#pragma unroll
    for (int b = 0; b < HD / 32; ++b)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        if (32 * b + 8 * g + 4 * (lane >> 5) < d)
          *(float4*)(p + 32 * b + 8 * g) = make_float4(acc[b][4 * g] * mul, acc[b][4 * g + 1] * mul,
                                                       acc[b][4 * g + 2] * mul, acc[b][4 * g + 3] * mul);
  }
};

template <class T, bool BIAS>
struct AttnOp {
  using E = typename T::E;
  using Rows = typename T::Rows;
  using Offs = typename T::Offs;
  using Src = typename T::Src;
  static constexpr int HD = T::HD, NB = HD / 32, TILE = T::TILE;
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
  // Entry e holds the bias (base 2) of distance j - i = e - off.  A near block
  // of 64 by 128 tokens reaches at most 190 tokens beyond `far`.
  static __device__ __forceinline__ int table_off(const AttnOpArgs& p) { return p.far + 192; }
  static __device__ __forceinline__ int table_len(const AttnOpArgs& p) { return 2 * p.far + 384; }
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
  // additions and three LDS atomics for 16 elements; the 16 atomics without the
  // shifts cost half of the kernel (us, dq of 13B's heads at s 4096, window
  // 2048, 64 buckets: DIAG).
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
  static __device__ __forceinline__ void add_diagonals(float* to, const f32x16& x) {
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
    __hip_atomic_fetch_add(to, s0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    __hip_atomic_fetch_add(to + 16, s1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    __hip_atomic_fetch_add(to + 32, s2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
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
  // key tiles of 64 for the queries [q0, q1]
  static __device__ __forceinline__ Steps key_steps(const AttnOpArgs& p, int q0, int q1, int len) {
    Steps s;
    q1 = min(q1, len - 1);
    if (q1 < q0) return {0, 0, 0};
    const int lo = max(0, q0 - p.left), hi = min((long)len - 1, (long)q1 + p.right);
    const int ns = p.causal ? min(p.sinks, q1 + 1) : min(p.sinks, len);
    const int nts = (ns + 63) / 64;
    s.t0 = lo / 64;
    s.n1 = min(nts, s.t0);
    s.n = s.n1 + max(hi / 64, nts - 1) - s.t0 + 1;
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
  // Lane column = key kk, elements = the queries q + 4 hh + row_of(r).
  static __device__ __forceinline__ void query_range(int& lo, unsigned& w, int q, int kk, int lane, int len,
                                                     const AttnOpArgs& p) {
    const int at = q + 4 * (lane >> 5);
    const bool sink = kk < p.sinks;
    lo = (int)max(0L, sink && !p.causal ? 0L : (long)kk - p.right) - at;
    int hi = (int)(sink ? (long)len - 1 : min((long)len - 1, (long)kk + p.left)) - at;
    if (kk >= len) hi = lo - 1;
    if (hi < lo) lo = 1 << 29, hi = lo;
    w = (unsigned)(hi - lo);
  }

  // body(stage, it) for n steps, whose operands issue(stage, it) copies: the next
  // step's while this one computes, or (copies through registers) its own.  The
  // caller has issued step 0 in the first case.
  static constexpr int STAGES = T::ASYNC ? 2 : 1;
  template <class Issue, class Body>
  static __device__ __forceinline__ void pipeline(int n, char* lds, int stage, Issue issue, Body body) {
    stage_sync();
    for (int it = 0; it < n; ++it) {
      if constexpr (T::ASYNC) {
        char* const cur = lds + (it & 1) * stage;
        if (it + 1 < n) issue(lds + (~it & 1) * stage, it + 1);
        body(cur, it);
        stage_sync();
      } else {
        issue(lds, it);
        stage_sync();
        body(lds, it);
        __syncthreads();
      }
    }
  }

  // -- forward -----------------------------------------------------------------
  struct Fwd {
    f32x16 o[NB];
    float m, l;
  };
  static __device__ __forceinline__ void fwd_tile(Fwd& st, const Rows& qf, const char* kt, const char* vt, const Offs& of,
                                                  int k0, int q0, int qq, int lane, int len, const float* table,
                                                  const AttnOpArgs& p) {
    if (none_visible<64>(p, q0, k0, len)) return;
    f32x16 sc[2];
    zero(sc[0]);
    zero(sc[1]);
    T::score2(sc[0], kt, 0, qf, sc[1], kt, 1, qf, of, lane);
    if constexpr (BIAS) {
      const int rel = k0 - q0;
      const bool near = wave_uniform(rel + 63 > -p.far && rel - 31 < p.far);
      const int e = k0 + 4 * (lane >> 5) - qq + table_off(p);
      float c = 0.f;
      if (!near) c = rel < 0 ? table[0] : table[table_len(p) - 1];
#pragma unroll
      for (int j = 0; j < 2; ++j) add_bias<1>(sc[j], table, e + 32 * j, c, near, p);
    }
    if (wave_uniform(!all_visible<32, 64>(p, q0, k0, len))) {
      mask_keys(sc[0], k0, qq, lane, -INFINITY, len, p);
      mask_keys(sc[1], k0 + 32, qq, lane, -INFINITY, len, p);
    }
    float mx = -INFINITY;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[j][r]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    if constexpr (!BIAS) mx *= p.sl2;
    // the reference moves when a row's maximum exceeds it by more than 2^8
    const bool grow = mx > st.m + 8.f;
    if (__any(grow)) {
      const float m_new = grow ? mx : st.m;
      const float alpha = __builtin_amdgcn_exp2f(st.m - m_new);
      st.m = m_new;
      st.l *= alpha;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) st.o[b][r] *= alpha;
    }
    float ls = 0.f;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float e = __builtin_amdgcn_exp2f(BIAS ? sc[j][r] - st.m : fmaf(sc[j][r], p.sl2, -st.m));
        sc[j][r] = e;
        ls += e;
      }
    st.l += ls;
    T::outer(st.o, vt, 0, sc[0], of, lane);
    T::outer(st.o, vt, 1, sc[1], of, lane);
  }

  static constexpr int STAGE = 2 * TILE;

  static __device__ __forceinline__ void fwd(const AttnOpArgs& p, char* lds) {
    float* const table = (float*)(lds + STAGES * STAGE);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int bh = p.batch * p.heads, nqb = (p.s + 127) / 128;
    const int z = blockIdx.x % bh, qb = nqb - 1 - blockIdx.x / bh;
    const int b = z / p.heads, h = z % p.heads;
    const int len = length(p, b);
    const int q0 = qb * 128 + 32 * wave, qq = q0 + (lane & 31);
    const Steps steps = key_steps(p, qb * 128, qb * 128 + 127, len);
    Src ks, vs;
    ks.set(base(p.k, b, h / p.group), p.k.t, len);
    vs.set(base(p.v, b, h / p.group), p.v.t, len);
    auto issue = [&](char* t, int it) {
      const int k0 = steps.tile(it) * 64;
      T::copy(t, ks, wave, lane, k0, len, p.d);
      T::copy(t + TILE, vs, wave, lane, k0, len, p.d);
    };
    if (T::ASYNC && steps.n > 0) issue(lds, 0);
    Rows qf;
    T::rows(qf, base(p.q, b, h), p.q.t, qq, len, lane, p.d);
    if constexpr (BIAS) fill_table(p, h, table);
    Offs of;
    of.init(lane);
    Fwd st;
#pragma unroll
    for (int i = 0; i < NB; ++i) zero(st.o[i]);
    st.m = kNone;
    st.l = 0.f;
    pipeline(steps.n, lds, STAGE, issue, [&](char* cur, int it) {
      fwd_tile(st, qf, cur, cur + TILE, of, steps.tile(it) * 64, q0, qq, lane, len, table, p);
    });
    // rows without a visible token: zeros
    const float l = st.l + __shfl_xor(st.l, 32, 64);
    const float inv = l > 0.f ? 1.0f / l : (l == l ? 0.f : l);
    if (qq >= len) {
#pragma unroll
      for (int i = 0; i < NB; ++i) zero(st.o[i]);
    }
    char* const area = lds + wave * (STAGE / 4);
    T::store(st.o, area, out(p.o, b, h), p.o.t, q0, p.s, lane, inv, p.d);
    if (!p.m) return;
    if constexpr (T::REST) {
#pragma unroll
      for (int i = 0; i < NB; ++i) T::A::keep_rest(st.o[i], inv);
      T::store(st.o, area, (E*)p.rest + ((long)b * p.s * p.heads + h) * p.d, (long)p.heads * p.d, q0, p.s, lane, 1.0f,
               p.d);
    }
    if (lane < 32 && qq < p.spad) {
      const bool some = l > 0.f || l != l;
      p.m[(long)z * p.spad + qq] = some ? st.m : 0.f;
      p.l[(long)z * p.spad + qq] = some ? __builtin_amdgcn_logf(l) : 0.f;
    }
  }

  // -- dq, dbias and D -----------------------------------------------------------
  // P of a score block in place; x: after add_bias with BIAS, raw products otherwise.
  static __device__ __forceinline__ float prob(float x, float m, float l, const AttnOpArgs& p) {
    return __builtin_amdgcn_exp2f((BIAS ? x - m : fmaf(x, p.sl2, -m)) - l);
  }

  static __device__ __forceinline__ void dq(const AttnOpArgs& p, char* lds) {
    float* const table = (float*)(lds + STAGES * STAGE);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int bh = p.batch * p.heads, nqb = (p.s + 127) / 128;
    const int z = blockIdx.x % bh, qb = nqb - 1 - blockIdx.x / bh;
    const int b = z / p.heads, h = z % p.heads;
    const int len = length(p, b);
    const int q0 = qb * 128 + 32 * wave, qq = q0 + (lane & 31);
    const Steps steps = key_steps(p, qb * 128, qb * 128 + 127, len);
    Src ks, vs;
    ks.set(base(p.k, b, h / p.group), p.k.t, len);
    vs.set(base(p.v, b, h / p.group), p.v.t, len);
    auto issue = [&](char* t, int it) {
      const int k0 = steps.tile(it) * 64;
      T::copy(t, ks, wave, lane, k0, len, p.d);
      T::copy(t + TILE, vs, wave, lane, k0, len, p.d);
    };
    if (T::ASYNC && steps.n > 0) issue(lds, 0);
    Rows qf, df;
    T::rows(qf, base(p.q, b, h), p.q.t, qq, len, lane, p.d);
    T::rows(df, base(p.dout, b, h), p.dout.t, qq, len, lane, p.d);
    float D = 0.f;
    {
      f32x16 a;
      zero(a);
      Rows of;
      T::rows(of, base(p.o, b, h), p.o.t, qq, len, lane, p.d);
      T::dot(a, of, df);
      if constexpr (T::REST) {
        T::rows(of, (const E*)p.rest + ((long)b * p.s * p.heads + h) * p.d, (long)p.heads * p.d, qq, len, lane, p.d);
        T::dot(a, of, df);
      }
      // the diagonal: row lane % 32 of column lane % 32, held by one half of the wave
      const int want = (lane & 31) - 4 * (lane >> 5);
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (row_of(r) == want) D = a[r];
      const bool mine = ((lane >> 2) & 1) == (lane >> 5);
      D = mine ? D : 0.f;
      D += __shfl_xor(D, 32, 64);
    }
    if (lane < 32 && qq < p.spad) p.drow[(long)z * p.spad + qq] = qq < len ? D : 0.f;
    const float m = qq < p.s ? p.m[(long)z * p.spad + qq] : 0.f;
    const float l = qq < p.s ? p.l[(long)z * p.spad + qq] : 0.f;
    // this half-wave's sums by distance, and those of far blocks on either side
    float* sums = nullptr;
    float far_l = 0.f, far_r = 0.f;
    if constexpr (BIAS) {
      fill_table(p, h, table);
      float* const all = table + table_len(p);
      for (int e = threadIdx.x; e < 8 * table_len(p); e += 256) all[e] = 0.f;
      sums = all + (2 * wave + (lane >> 5)) * table_len(p);
    }
    Offs of;
    of.init(lane);
    f32x16 acc[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) zero(acc[i]);
    pipeline(steps.n, lds, STAGE, issue, [&](char* cur, int it) {
      const int k0 = steps.tile(it) * 64;
#pragma unroll 1
      for (int j = 0; j < 2; ++j) {
        const int k = k0 + 32 * j;
        if (none_visible<32>(p, q0, k, len)) continue;
        f32x16 sc, dp;
        zero(sc);
        zero(dp);
        T::score2(sc, cur, j, qf, dp, cur + TILE, j, df, of, lane);
        const int rel = k - q0;
        const bool near = BIAS && wave_uniform(rel + 31 > -p.far && rel - 31 < p.far);
        const int e = k + 4 * (lane >> 5) - qq + (BIAS ? table_off(p) : 0);
        if constexpr (BIAS) {
          float c = 0.f;
          if (!near) c = rel < 0 ? table[0] : table[table_len(p) - 1];
          add_bias<1>(sc, table, e, c, near, p);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = prob(sc[r], m, l, p);
        if (wave_uniform(!all_visible<32, 32>(p, q0, k, len))) mask_keys(sc, k, qq, lane, 0.f, len, p);
#pragma unroll
        for (int r = 0; r < 16; ++r) dp[r] = sc[r] * (dp[r] - D);
        if constexpr (BIAS) {
          if (near) {
            add_diagonals(sums + e, dp);
          } else {
            float t = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) t += dp[r];
            if (rel < 0)
              far_l += t;
            else
              far_r += t;
          }
        }
        T::outer(acc, cur, j, dp, of, lane);
      }
    });
    if (qq >= len) {
#pragma unroll
      for (int i = 0; i < NB; ++i) zero(acc[i]);
    }
    T::store(acc, lds + wave * (STAGE / 4), out(p.dq, b, h), p.dq.t, q0, p.s, lane, p.scale, p.d);
    if constexpr (BIAS) {
      // eight tables into one, in order, then the sums of each bucket
      const int n = table_len(p), off = table_off(p);
      float* const all = table + n;
      float* const fars = table;  // the bias is no longer needed
      far_l = wave_sum(far_l);
      far_r = wave_sum(far_r);
      if (lane == 0) fars[wave] = far_l, fars[4 + wave] = far_r;
      for (int e = threadIdx.x; e < n; e += 256) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) t += all[i * n + e];
        all[e] = t;
      }
      __syncthreads();
      const int side = p.causal ? p.buckets : p.buckets / 2;
      float* const to = p.bpart + ((long)z * nqb + qb) * p.buckets;
      for (int c = wave; c < p.buckets; c += 4) {
        const bool ahead = c >= side;
        const int cs = ahead ? c - side : c;
        // its distances [n0, n1); distance 0 counts once
        const int n0 = max((int)p.first[cs], ahead ? 1 : 0);
        const int n1 = cs == side - 1 ? off : p.first[cs + 1];
        float t = 0.f;
        for (int e = n0 + lane; e < n1; e += 64) t += all[ahead ? off + e : off - e];
        t = wave_sum(t);
        if (cs == side - 1) {
          const float* f = fars + (ahead ? 4 : 0);
          t += f[0] + f[1] + f[2] + f[3];
        }
        if (lane == 0) to[c] = t;
      }
    }
  }

  // -- dk and dv -------------------------------------------------------------------
  // A stage: a Q tile, a dO tile and the row vectors m, l, D of 64 queries.
  static constexpr int KSTAGE = 2 * TILE + 3072;

  static __device__ __forceinline__ void dkv(const AttnOpArgs& p, char* lds) {
    float* const table = (float*)(lds + STAGES * KSTAGE);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int bk = p.batch * p.kv_heads, z = blockIdx.x % bk, u = blockIdx.x / bk;
    const int b = z / p.kv_heads, hk = z % p.kv_heads;
    const int len = length(p, b);
    const int units = p.sink_blocks * p.chunks;
    const int kb = u < units ? u / p.chunks : u - units + p.sink_blocks;
    const int K0 = kb * 128, k0 = K0 + 32 * wave, kk = k0 + (lane & 31);
    // the queries of this workgroup
    int qlo, qhi;
    if (u < units) {
      const int c = u % p.chunks;
      qlo = max(p.causal ? K0 : 0, c * p.chunk_len);
      qhi = min(len, (c + 1) * p.chunk_len) - 1;
    } else {
      qlo = (int)max(0L, (long)K0 - p.right);
      qhi = (int)min((long)len - 1, (long)K0 + 127 + p.left);
    }
    if (K0 >= len) qhi = -1;
    const int t0 = qlo / 64, nt = qhi >= qlo ? qhi / 64 - t0 + 1 : 0;
    Src qs, ds;
    // step i: tile i % nt of head i / nt of the group; steps are issued and
    // computed in order, so both count along
    int gi = 0, ti = 0, gc = 0, tc = 0;
    auto issue = [&](char* t, int) {
      const int h = hk * p.group + gi, row0 = (t0 + ti) * 64;
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
    if (T::ASYNC && nt > 0) issue(lds, 0);
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
    pipeline(nt * p.group, lds, KSTAGE, issue, [&](char* cur, int) {
      if constexpr (BIAS) {
        if (tc == 0) {  // the first tile of a head: its bias
          fill_table(p, hk * p.group + gc, table);
          __syncthreads();
        }
      }
      const int q64 = (t0 + tc) * 64;
      const float* vec = (const float*)(cur + 2 * TILE);
#pragma unroll 1
      for (int j = 0; j < 2; ++j) {
        const int q = q64 + 32 * j;
        if (none_visible<32>(p, q, k0, len)) continue;
        f32x16 sc, dp;
        zero(sc);
        zero(dp);
        T::score2(sc, cur, j, kf, dp, cur + TILE, j, vf, of, lane);
        if constexpr (BIAS) {
          const int rel = k0 - q;
          const bool near = wave_uniform(rel + 31 > -p.far && rel - 31 < p.far);
          float c = 0.f;
          if (!near) c = rel < 0 ? table[0] : table[table_len(p) - 1];
          add_bias<-1>(sc, table, kk - q - 4 * (lane >> 5) + table_off(p), c, near, p);
        }
        const float* row = vec + 32 * j + 4 * (lane >> 5);
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = prob(sc[r], row[row_of(r)], row[256 + row_of(r)], p);
        if (wave_uniform(!all_visible<32, 32>(p, q, k0, len))) {
          int lo;
          unsigned w;
          query_range(lo, w, q, kk, lane, len, p);
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if ((unsigned)(row_of(r) - lo) > w) sc[r] = 0.f;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) dp[r] = sc[r] * (dp[r] - row[512 + row_of(r)]);
        T::outer(dv, cur + TILE, j, sc, of, lane);
        T::outer(dk, cur, j, dp, of, lane);
      }
      if (++tc == nt) tc = 0, ++gc;
    });
    if (kk >= len) {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        zero(dk[i]);
        zero(dv[i]);
      }
    }
    if (u < units && p.chunks > 1) {
      float* to = p.spart + (((long)z * units + u) * 2 * 128 + 32 * wave + (lane & 31)) * HD + 4 * (lane >> 5);
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          *(float4*)(to + 32 * i + 8 * c) =
              make_float4(dk[i][4 * c], dk[i][4 * c + 1], dk[i][4 * c + 2], dk[i][4 * c + 3]);
          *(float4*)(to + 128L * HD + 32 * i + 8 * c) =
              make_float4(dv[i][4 * c], dv[i][4 * c + 1], dv[i][4 * c + 2], dv[i][4 * c + 3]);
        }
      return;
    }
    char* const area = lds + wave * (STAGE / 4);
    T::store(dk, area, out(p.dk, b, hk), p.dk.t, k0, p.s, lane, p.scale, p.d);
    T::store(dv, area, out(p.dv, b, hk), p.dv.t, k0, p.s, lane, 1.0f, p.d);
  }
};

// Key blocks with sinks: dk and dv from their chunks' shares, in order.  One
// workgroup per sequence, key head and 8 keys; a thread sums 4 columns.
template <class T>
__global__ __launch_bounds__(256) void attn_op_sinks_k(AttnOpArgs p) {
  constexpr int HD = T::HD, C4 = HD / 4;
  const int bk = p.batch * p.kv_heads, z = blockIdx.x % bk, r8 = blockIdx.x / bk;
  const int b = z / p.kv_heads, h = z % p.kv_heads;
  for (int i = threadIdx.x; i < 8 * 2 * C4; i += 256) {
    const int c = 4 * (i % C4), which = i / C4 % 2, row = 8 * r8 + i / (2 * C4);
    const int kb = row / 128;
    if (row >= p.s || c >= p.d) continue;
    const float* src = p.spart + ((((long)z * p.sink_blocks + kb) * p.chunks * 2 + which) * 128 + row % 128) * HD + c;
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int n = 0; n < p.chunks; ++n) {
      const float4 v = *(const float4*)(src + (long)n * 2 * 128 * HD);
      t.x += v.x;
      t.y += v.y;
      t.z += v.z;
      t.w += v.w;
    }
    const float mul = which ? 1.0f : p.scale;
    const AttnOpView& v = which ? p.dv : p.dk;
    typename T::E* o = (typename T::E*)v.p + (long)b * v.b + (long)row * v.t + (long)h * v.h + c;
    typename T::E w[4] = {(typename T::E)(t.x * mul), (typename T::E)(t.y * mul), (typename T::E)(t.z * mul),
                          (typename T::E)(t.w * mul)};
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = w[e];
  }
}

extern __shared__ __attribute__((aligned(1024))) char attn_op_lds[];

template <class T, bool BIAS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(T::WAVES, T::WAVES))) void attn_op_fwd_k(
    AttnOpArgs p) {
  AttnOp<T, BIAS>::fwd(p, attn_op_lds);
}
template <class T, bool BIAS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(T::WAVES, T::WAVES))) void attn_op_dq_k(
    AttnOpArgs p) {
  AttnOp<T, BIAS>::dq(p, attn_op_lds);
}
template <class T, bool BIAS>
__global__ __launch_bounds__(256) void attn_op_dkv_k(AttnOpArgs p) {
  AttnOp<T, BIAS>::dkv(p, attn_op_lds);
}

template <class T>
hipError_t attn_op_fwd_launch(const AttnOpArgs& a, hipStream_t st) {
  using K = AttnOp<T, false>;
  const dim3 grid((unsigned)((a.s + 127) / 128 * (long)a.batch * a.heads));
  const size_t table = a.bias ? 4 * (2 * (size_t)a.far + 384) : 0;
  if (a.bias)
    hipLaunchKernelGGL((attn_op_fwd_k<T, true>), grid, dim3(256), K::STAGES * K::STAGE + table, st, a);
  else
    hipLaunchKernelGGL((attn_op_fwd_k<T, false>), grid, dim3(256), K::STAGES * K::STAGE, st, a);
  return hipGetLastError();
}

template <class T>
hipError_t attn_op_bwd_launch(const AttnOpArgs& a, hipStream_t st) {
  using K = AttnOp<T, false>;
  const long nb = (a.s + 127) / 128;
  const size_t table = a.bias ? 4 * (2 * (size_t)a.far + 384) : 0;
  const dim3 gq((unsigned)(nb * a.batch * a.heads));
  const dim3 gk((unsigned)((nb + (long)a.sink_blocks * (a.chunks - 1)) * a.batch * a.kv_heads));
  if (a.bias) {
    hipLaunchKernelGGL((attn_op_dq_k<T, true>), gq, dim3(256), K::STAGES * K::STAGE + 9 * table, st, a);
    hipLaunchKernelGGL((attn_op_dkv_k<T, true>), gk, dim3(256), K::STAGES * K::KSTAGE + table, st, a);
  } else {
    hipLaunchKernelGGL((attn_op_dq_k<T, false>), gq, dim3(256), K::STAGES * K::STAGE, st, a);
    hipLaunchKernelGGL((attn_op_dkv_k<T, false>), gk, dim3(256), K::STAGES * K::KSTAGE, st, a);
  }
  if (a.sink_blocks && a.chunks > 1) {
    const long rows = a.sink_blocks * 128L < a.s ? a.sink_blocks * 128L : a.s;
    hipLaunchKernelGGL((attn_op_sinks_k<T>), dim3((unsigned)((rows + 7) / 8 * a.batch * a.kv_heads)), dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace
