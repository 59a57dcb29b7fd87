// Attention of few new rows over a paged cache (the next event of each user, a handful of them), and the sum of the parts of
// cut tiles.
//
//   O_i = (1 / N) sum over the visible cached rows j of silu(alpha (q_i . k_j [+ w(i, j)])) v_j
//
// One new row reads every cached key and value of its sequence once and does 4 d flops per row of 4 d bytes (bf16): the pass is
// bound by reading the cache, and everything here serves to keep loads in flight.
//   - A wave is a worker of its own (no LDS, no barrier): it takes a run of the line of all work (hstu_paged.h) and streams
//     blocks of keys through registers, the next block's loads issued before the present one is used: at d = 128 a
//     block of 16 KB per wave, 64 KB in flight per CU with a worker per SIMD.
//   - 16 (new row, query head) pairs that share a key/value head are one operand of the 16x16 matrix instructions: query heads
//     that share keys, and a few new rows, cost no further reads.  One pair alone leaves 15 columns unused: the matrix pipe
//     then still has 5 times the throughput that the loads can feed.
//   - S^T = K Q^T leaves P^T in the accumulators as the second product's operand (its contraction index is
//     matched to them by the choice of the rows a lane loads), and V's rows are loaded whole, 16 bytes per lane, and transposed
//     inside the lane (one byte permutation per register): nothing goes through LDS.
//   - P enters the second product as two bf16 terms, whose sum is exact to 2^-17 of it, for 8 more matrix instructions per block
//     in a loop that waits for memory: the result is off by its own rounding alone.  Two terms of opposite signs make NaN of an infinite
//     value, and an infinite P has no second term, so a tile whose sums end up infinite or NaN is streamed once more, in a form that
//     takes such terms apart (FewBf16::careful_values): what is finite, which is nearly everything, pays a test per tile.
//   - Rows behind the part's end and rows of pages that do not exist lie outside the buffer descriptors: they arrive as zeros
//     without traffic, so what such memory holds (other users' rows, NaN) has no way in.
#include "hstu_mfma.h"
#include "hstu_paged.h"

namespace hstu {

namespace {

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;

// Descriptor of `rows` rows (of `row_bytes`) from p on; loads beyond them return zero.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const char* p, int rows, int row_bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, rows * row_bytes, 0x00020000);
}

// AUX 2: nontemporal (see PagedArgs::stream).
template <int W, int AUX>
__device__ __forceinline__ void load_words(uint32_t (&dst)[W], __amdgpu_buffer_rsrc_t r, int voff) {
  if constexpr (W == 4) {
    const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(r, voff, 0, AUX);
#pragma unroll
    for (int i = 0; i < 4; ++i) dst[i] = x[i];
  } else if constexpr (W == 2) {
    const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(r, voff, 0, AUX);
    dst[0] = x[0]; dst[1] = x[1];
  } else {
    dst[0] = __builtin_amdgcn_raw_buffer_load_b32(r, voff, 0, AUX);
  }
}

// What a block of a tile's stream needs besides its own keys.
struct TileCtx {
  int lim;       // keys the lane's pair sees
  int lim0, vis; // ... the tile's first and last row see
  int tq;        // the lane's pair's timestamp
  float c1;      // -alpha log2 e
  const float* wtab;
  int nb, f;
};

// Where 16 rows of one page are: keys [key, key + 16) of a sequence, for one head.
struct Rows16 {
  const char* k;
  const char* v;
  const int32_t* ts;
  int n;         // rows of them that belong to the part (0: none, or no such page)
};
template <int ROW_K, int ROW_V>
__device__ __forceinline__ Rows16 rows16(const PagedView& c, const PageIds& ids, int h, int key, int end) {
  const int id = ids.get(key >> c.ps_log2);
  const int slot = key & ((1 << c.ps_log2) - 1);
  Rows16 r;
  const int64_t row = ((int64_t)h << c.ps_log2) + slot, page = id < 0 ? 0 : id;
  r.k = c.k + page * c.k_page + row * ROW_K;
  r.v = c.v + page * c.v_page + row * ROW_V;
  r.ts = c.ts + (page << c.ps_log2) + slot;
  r.n = rows_before(id, key, end, 16);
  return r;
}

// ---- bf16 ----------------------------------------------------------------------------------------------------------------
//   v_mfma_f32_16x16x32_bf16  D[16x16] += A[16x32] B[32x16]   (lane l: i = l % 16, g = l / 16)
//     A: lane holds row i, k = 8 g .. 8 g + 7     B: column i, same k     D: column i, rows 4 g + r, r = 0..3
// Block of 32 keys: two S^T products (keys 0..15 and 16..31 as rows), whose accumulators hold for the lane's pair the keys
// 4 g + r and 16 + 4 g + r; those eight are the contraction index 8 g .. 8 g + 7 of the second product, so lane (i, g) loads
// these eight rows of V, at elements VE * i .. of each (VE = d_v / 16), and product e of VE makes the output's elements VE * row + e.
template <int DQK, int DV, bool BIAS, int AUX>
struct FewBf16 {
  static constexpr int BK = 32, PARTS = 2, KS = DQK / 32, VE = DV / 16, VW = VE / 2;
  static constexpr int ROW_K = DQK * 2, ROW_V = DV * 2;
  struct Block {
    uint32_t k[2][KS][4];
    uint32_t v[8][VW];
    uint32_t ts[2][4];
  };
  Block b;
  bf16x8 q[KS];
  f32x4 acc[VE];
  int ko, vo, to;  // the lane's byte offsets inside 16 rows

  __device__ __forceinline__ void init() {
    const int i = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
    ko = i * ROW_K + g * 16;
    vo = 4 * g * ROW_V + i * VE * 2;
    to = 16 * g;
  }
  __device__ __forceinline__ void start(const char* qrow) {  // qrow: the lane's pair's row, or null
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      u32x4 z = {0, 0, 0, 0};
      if (qrow) z = *(const u32x4*)(qrow + ks * 64 + g * 16);
      q[ks] = __builtin_bit_cast(bf16x8, z);
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ void where(Rows16 (&r)[PARTS], const PagedView& c, const PageIds& ids, int h, int key, int end) const {
#pragma unroll
    for (int x = 0; x < 2; ++x) r[x] = rows16<ROW_K, ROW_V>(c, ids, h, key + 16 * x, end);
  }
  __device__ __forceinline__ void fetch_k(const Rows16 (&r)[PARTS]) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const __amdgpu_buffer_rsrc_t rk = rows_rsrc(r[x].k, r[x].n, ROW_K);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) load_words<4, AUX>(b.k[x][ks], rk, ko + ks * 64);
      if constexpr (BIAS) load_words<4, AUX>(b.ts[x], rows_rsrc((const char*)r[x].ts, r[x].n, 4), to);
    }
  }
  __device__ __forceinline__ void fetch_v(const Rows16 (&r)[PARTS]) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const __amdgpu_buffer_rsrc_t rv = rows_rsrc(r[x].v, r[x].n, ROW_V);
#pragma unroll
      for (int e = 0; e < 4; ++e) load_words<VW, AUX>(b.v[4 * x + e], rv, vo + e * ROW_V);
    }
  }
  // V's operand of output elements VE * row + e, rows behind `lim` of the block's keys left out where CUT.
  template <bool CUT>
  __device__ __forceinline__ bf16x8 v_operand(int e, int lim, int g) const {
    u32x4 w;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      uint32_t lo = b.v[2 * p][e >> 1], hi = b.v[2 * p + 1][e >> 1];
      if constexpr (CUT) {
        const int key = (p >> 1) * 16 + 4 * g + 2 * (p & 1);
        lo = key < lim ? lo : 0;
        hi = key + 1 < lim ? hi : 0;
      }
      w[p] = __builtin_amdgcn_perm(hi, lo, (e & 1) ? 0x07060302 : 0x05040100);
    }
    return __builtin_bit_cast(bf16x8, w);
  }
  float p[8];
  __device__ __forceinline__ void scores(const TileCtx& t) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
      if constexpr (BIAS)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[r] = t.wtab[bias_bucket(abs_diff(t.tq, (int)b.ts[x][r]), t.nb, t.f)];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const u32x4 z = {b.k[x][ks][0], b.k[x][ks][1], b.k[x][ks][2], b.k[x][ks][3]};
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, z), q[ks], s, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) p[4 * x + r] = s[r];
    }
  }
  template <bool CAREFUL>
  __device__ __forceinline__ void values(const TileCtx& t, int key) {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] *= sigmoid_scaled(p[e], t.c1);
    const bool masked = t.lim0 < t.vis && key + BK > t.lim0;
    if (masked) {
      asm volatile("" ::: "memory");
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = key + (e >> 2) * 16 + 4 * g + (e & 3) < t.lim ? p[e] : 0.f;
    }
    if constexpr (CAREFUL) {
      careful_values(t, key, masked);
      return;
    }
    bf16x8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      hi[e] = (__bf16)p[e];
      lo[e] = (__bf16)(p[e] - (float)hi[e]);
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const bf16x8 v = v_operand<false>(e, 0, g);
      acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, hi, acc[e], 0, 0, 0);
      acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, lo, acc[e], 0, 0, 0);
    }
  }
  // The same where values or probabilities are infinite or NaN.  An infinite P has no second term, one that only rounds to infinity keeps
  // the largest finite bf16 as its first; an infinite or NaN value is multiplied by the first term alone.  In a masked block, which
  // some pairs see more of than others, such a value times a zero of P would reach the pairs that do not see it: the block is
  // multiplied once per row position, without the rows behind it.
  __device__ __forceinline__ void careful_values(const TileCtx& t, int key, bool masked) {
    const int g = (threadIdx.x & 63) >> 4;
    bf16x8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool finite = __builtin_fabsf(p[e]) <= 0x1.fffffep127f;
      const float most = 0x1.fep127f;  // the largest finite bf16
      const float h = finite ? __builtin_fminf(__builtin_fmaxf(p[e], -most), most) : p[e];
      hi[e] = (__bf16)h;
      lo[e] = (__bf16)(finite ? p[e] - (float)hi[e] : 0.f);
    }
    for (int lim = masked ? t.lim0 : t.vis; lim <= t.vis; ++lim) {
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const bf16x8 v = v_operand<true>(e, masked ? lim - key : BK, g);
        u32x4 f = __builtin_bit_cast(u32x4, v);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t low = (f[w] & 0x7f80u) == 0x7f80u ? 0u : f[w] & 0xffffu;
          f[w] = low | ((f[w] & 0x7f800000u) == 0x7f800000u ? 0u : f[w] & 0xffff0000u);
        }
        f32x4 part = acc[e];
        part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, hi, part, 0, 0, 0);
        part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), lo, part, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[e][r] = !masked || t.lim == lim ? part[r] : acc[e][r];
      }
    }
  }
  // Has any of the wave's pairs an infinite or NaN sum?  (No such term can leave the sum finite again.)
  __device__ __forceinline__ bool lost() const {
    float z = 0.f;
#pragma unroll
    for (int e = 0; e < VE; ++e)
#pragma unroll
      for (int r = 0; r < 4; ++r) z = __builtin_fmaf(acc[e][r], 0.f, z);
    return __ballot(z != 0.f) != 0;
  }
  // The lane's part of its pair's output row: elements 4 VE g .. + 4 VE - 1.
  __device__ __forceinline__ void result(float (&x)[4 * VE]) const {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < VE; ++e) x[r * VE + e] = acc[e][r];
  }
  static constexpr int OUT = 4 * VE;
};

// ---- fp32 ----------------------------------------------------------------------------------------------------------------
//   v_mfma_f32_16x16x4_f32  D[16x16] += A[16x4] B[4x16]: A lane holds row i, k = g; B column i, same k; D as above.
// Block of 16 keys.  The contraction over d_qk takes element 16 s + 4 g + e of a row at step (s, e); the one over keys takes key
// 4 g + r at step r, which is what accumulator register r holds; lane (i, g) loads V's rows 4 g + r at elements
// 16 VE j + VE i .. (VE = min(4, d_v / 16)), and product (j, e) makes the output's elements 16 VE j + VE * row + e.
template <int DQK, int DV, bool BIAS, int AUX>
struct FewF32 {
  static constexpr int BK = 16, PARTS = 1, KS = DQK / 16, VE = DV >= 64 ? 4 : 2, NJ = DV / (16 * VE);
  static constexpr int ROW_K = DQK * 4, ROW_V = DV * 4;
  struct Block {
    uint32_t k[KS][4];
    uint32_t v[4][NJ][VE];
    uint32_t ts[4];
  };
  Block b;
  float q[KS][4];
  f32x4 acc[NJ][VE];
  int ko, vo, to;

  __device__ __forceinline__ void init() {
    const int i = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
    ko = i * ROW_K + g * 16;
    vo = 4 * g * ROW_V + i * VE * 4;
    to = 16 * g;
  }
  __device__ __forceinline__ void start(const char* qrow) {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
      if (qrow) z = *(const float4*)(qrow + s * 64 + g * 16);
      q[s][0] = z.x; q[s][1] = z.y; q[s][2] = z.z; q[s][3] = z.w;
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < VE; ++e) acc[j][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ void where(Rows16 (&r)[PARTS], const PagedView& c, const PageIds& ids, int h, int key, int end) const {
    r[0] = rows16<ROW_K, ROW_V>(c, ids, h, key, end);
  }
  __device__ __forceinline__ void fetch_k(const Rows16 (&r)[PARTS]) {
    const __amdgpu_buffer_rsrc_t rk = rows_rsrc(r[0].k, r[0].n, ROW_K);
#pragma unroll
    for (int s = 0; s < KS; ++s) load_words<4, AUX>(b.k[s], rk, ko + s * 64);
    if constexpr (BIAS) load_words<4, AUX>(b.ts, rows_rsrc((const char*)r[0].ts, r[0].n, 4), to);
  }
  __device__ __forceinline__ void fetch_v(const Rows16 (&r)[PARTS]) {
    const __amdgpu_buffer_rsrc_t rv = rows_rsrc(r[0].v, r[0].n, ROW_V);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int j = 0; j < NJ; ++j) load_words<VE, AUX>(b.v[e][j], rv, vo + e * ROW_V + j * 16 * VE * 4);
  }
  f32x4 s;
  __device__ __forceinline__ void scores(const TileCtx& t) {
    s = f32x4{0.f, 0.f, 0.f, 0.f};
    if constexpr (BIAS)
#pragma unroll
      for (int r = 0; r < 4; ++r) s[r] = t.wtab[bias_bucket(abs_diff(t.tq, (int)b.ts[r]), t.nb, t.f)];
    f32x4 s2 = {0.f, 0.f, 0.f, 0.f};  // (two chains of half the length: less latency, less rounding)
#pragma unroll
    for (int ks = 0; ks < KS; ks += 2)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, b.k[ks][e]), q[ks][e], s, 0, 0, 0);
        s2 = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, b.k[ks + 1][e]), q[ks + 1][e], s2, 0, 0, 0);
      }
#pragma unroll
    for (int r = 0; r < 4; ++r) s[r] += s2[r];
  }
  template <bool CAREFUL>
  __device__ __forceinline__ void values(const TileCtx& t, int key) {
    const int g = (threadIdx.x & 63) >> 4;
    float p[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) p[r] = s[r] * sigmoid_scaled(s[r], t.c1);
    const bool masked = t.lim0 < t.vis && key + BK > t.lim0;
    if (masked) {
      asm volatile("" ::: "memory");
      uint32_t bad = 0;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[r] = key + 4 * g + r < t.lim ? p[r] : 0.f;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int e = 0; e < VE; ++e) bad |= (uint32_t)((b.v[r][j][e] & 0x7f800000u) == 0x7f800000u);
      }
      // Values that some pairs see and others do not: an infinity or NaN there times a zero of P would reach the pairs that do not see
      // it, so such a block is multiplied once per row position, without the rows behind it.
      if (__ballot(bad != 0) != 0) {
        for (int lim = t.lim0; lim <= t.vis; ++lim)
#pragma unroll
          for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int e = 0; e < VE; ++e) {
              f32x4 part = acc[j][e];
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float v = key + 4 * g + r < lim ? __builtin_bit_cast(float, b.v[r][j][e]) : 0.f;
                part = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[r], part, 0, 0, 0);
              }
#pragma unroll
              for (int r = 0; r < 4; ++r) acc[j][e][r] = t.lim == lim ? part[r] : acc[j][e][r];
            }
        return;
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < VE; ++e)
          acc[j][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, b.v[r][j][e]), p[r], acc[j][e], 0, 0, 0);
  }
  __device__ __forceinline__ void result(float (&x)[4 * VE * NJ]) const {
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int e = 0; e < VE; ++e) x[(j * 4 + r) * VE + e] = acc[j][e][r];
  }
  static constexpr int OUT = 4 * VE * NJ;
};

template <bool F32, int DQK, int DV, bool BIAS, int AUX>
using Few = typename std::conditional<F32, FewF32<DQK, DV, BIAS, AUX>, FewBf16<DQK, DV, BIAS, AUX>>::type;

// Element of the output row that the lane's value x of result() is.
template <bool F32, int DV>
__device__ __forceinline__ int out_element(int x, int g) {
  if constexpr (!F32) {
    return (DV / 4) * g + x;
  } else {
    constexpr int VE = DV >= 64 ? 4 : 2;
    const int j = x / (4 * VE), y = x % (4 * VE);
    return 16 * VE * j + 4 * VE * g + y;
  }
}

// Rounds and stores four neighbouring elements of an output row.
__device__ __forceinline__ void store4(const PagedArgs& a, int64_t elem, float x0, float x1, float x2, float x3) {
  const float scale = a.alpha * a.inv_n;
  if (a.out_f32) {
    *(float4*)((float*)a.o + elem) = make_float4(x0 * scale, x1 * scale, x2 * scale, x3 * scale);
  } else {
    bf16x4 z;
    z[0] = (__bf16)(x0 * scale); z[1] = (__bf16)(x1 * scale); z[2] = (__bf16)(x2 * scale); z[3] = (__bf16)(x3 * scale);
    *(bf16x4*)((__bf16*)a.o + elem) = z;
  }
}

// Streams the keys [k0, k1) of head h of sequence b past the wave's pairs.
template <bool CAREFUL, class F>
__device__ __forceinline__ void stream_keys(F& f, const PagedArgs& a, const TileCtx& t, int b, int h, int k0, int k1) {
  if (k0 >= k1) return;
  constexpr int BK = F::BK;
  PageIds ids;
  const int entries = (k1 + (1 << a.c.ps_log2) - 1) >> a.c.ps_log2;
  ids.fill(a.c, b, k0 >> a.c.ps_log2, entries);
  Rows16 r[F::PARTS];
  auto where = [&](int key) {  // (behind the part's end: rows of no length, so that every path issues the same loads)
    const bool more = key < k1;
    if (more && !ids.holds((key + BK - 1) >> a.c.ps_log2)) ids.fill(a.c, b, key >> a.c.ps_log2, entries);
    f.where(r, a.c, ids, h, more ? key : k0, more ? k1 : k0);
  };
  where(k0);
  f.fetch_k(r);
  f.fetch_v(r);
  // K of the next block is loaded once this one's scores are made, V once it has been multiplied: a block and a half in flight
  for (int key = k0; key < k1; key += BK) {
    f.scores(t);
    __builtin_amdgcn_sched_barrier(0);
    where(key + BK);
    f.fetch_k(r);
    __builtin_amdgcn_sched_barrier(0);
    f.template values<CAREFUL>(t, key);
    __builtin_amdgcn_sched_barrier(0);
    f.fetch_v(r);
  }
}

// NW = 1: workers are waves.  NW > 1: a worker is a workgroup whose waves share a tile's keys and add up their results in LDS.
template <bool F32, int DQK, int DV, bool BIAS, int NW, int AUX>
__global__ void __launch_bounds__(64 * NW, 2) paged_few_kernel(PagedArgs a) {
  typedef Few<F32, DQK, DV, BIAS, AUX> F;
  constexpr int ES = F32 ? 4 : 2;
  __shared__ float wtab[BIAS ? MAX_TS_BUCKETS : 1];
  __shared__ float4 sums[NW > 1 ? NW * FEW_PAIRS * DV / 4 : 1];
  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;

  Line<FEW_PAIRS> line;
  line.init(a);
  const int64_t share = share_of(a, line.total), active = uniform64(quotient(line.total + share - 1, share));
  const int64_t w = uniform64(worker_place(blockIdx.x, active));
  if (w >= active) {
    if (!a.whole && lane == 0) a.cut[w].parts = 0;
    return;
  }
  if constexpr (BIAS) {
    for (int x = threadIdx.x; x < a.nb; x += 64 * NW) wtab[x] = a.ts_w[x];
    __syncthreads();
  }
  int64_t at = w * share;
  const int64_t end = at + share < line.total ? at + share : line.total;
  Place pl = line.find(a, at);

  F f;
  f.init();
  TileCtx t;
  t.c1 = -a.alpha * 1.4426950408889634f;
  t.wtab = wtab;
  t.nb = a.nb;
  t.f = a.f;
  t.tq = 0;
  CutTile cut = {};
  while (at < end && pl.b < a.batch) {
    const Segment sg = make_segment<FEW_PAIRS>(a, pl.s, pl.t, pl.u, end - at);
    // the lane's pair
    const int pair = pl.t * FEW_PAIRS + i;
    const int row = pair / a.group, head = pl.h * a.group + pair % a.group;
    const bool on = i < sg.pairs;
    const int64_t qrow = pl.s.row0 + row;
    if constexpr (BIAS) t.tq = on ? a.ts_q[qrow] : 0;
    t.lim0 = sg.lim0;
    t.vis = sg.vis;
    t.lim = a.causal ? clampi((int64_t)pl.s.n - pl.s.m + row + 1, 0, pl.s.n) : pl.s.n;
    const char* const q = on ? a.q + qrow * a.q_stride + (int64_t)head * DQK * ES : nullptr;
    auto stream = [&](int k0, int k1) __attribute__((always_inline)) {
      f.start(q);
      stream_keys<false>(f, a, t, pl.b, pl.h, k0, k1);
      if constexpr (!F32)
        if (__builtin_expect(f.lost(), 0)) {
          f.start(q);
          stream_keys<true>(f, a, t, pl.b, pl.h, k0, k1);
        }
    };

    if constexpr (NW > 1) {
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
      const int per = ((sg.k1 + 32 * NW - 1) / (32 * NW)) * 32, k0 = wave * per;  // (whole tiles: from key 0 on)
      stream(k0, k0 + per < sg.k1 ? k0 + per : sg.k1);
      float x[F::OUT];
      f.result(x);
      float* slot = (float*)sums + (wave * FEW_PAIRS + i) * DV;
      if (on)
#pragma unroll
        for (int y = 0; y < F::OUT; y += 4)
          *(float4*)(slot + out_element<F32, DV>(y, g)) = make_float4(x[y], x[y + 1], x[y + 2], x[y + 3]);
      __syncthreads();
      for (int c = threadIdx.x; c < sg.pairs * (DV / 4); c += 64 * NW) {
        float4 s = sums[c];
#pragma unroll
        for (int v = 1; v < NW; ++v) {
          const float4 y = sums[v * FEW_PAIRS * DV / 4 + c];
          s.x += y.x; s.y += y.y; s.z += y.z; s.w += y.w;
        }
        const int p = pl.t * FEW_PAIRS + c / (DV / 4);
        const int64_t o = (int64_t)(pl.s.row0 + p / a.group) * a.heads + pl.h * a.group + p % a.group;
        store4(a, o * DV + (c % (DV / 4)) * 4, s.x, s.y, s.z, s.w);
      }
      return;  // (one tile)
    }

    stream(sg.k0, sg.k1);
    if (on) {
      float x[F::OUT];
      f.result(x);
      if (sg.first && sg.last) {
        const int64_t elem = (qrow * a.heads + head) * DV;
#pragma unroll
        for (int y = 0; y < F::OUT; y += 4)
          store4(a, elem + out_element<F32, DV>(y, g), x[y], x[y + 1], x[y + 2], x[y + 3]);
      } else {
        float* slot = a.partial + ((2 * w + (sg.first ? 1 : 0)) * FEW_PAIRS + i) * DV;
#pragma unroll
        for (int y = 0; y < F::OUT; y += 4)
          *(float4*)(slot + out_element<F32, DV>(y, g)) = make_float4(x[y], x[y + 1], x[y + 2], x[y + 3]);
      }
    }
    cut = cut_tile(a, pl, sg, at, share, w, FEW_PAIRS);
    at += sg.u1 - sg.u0;
    line.next(a, pl);
  }
  if (!a.whole && lane == 0) a.cut[w] = cut;
}

// ---- large batches: the lanes' sums -----------------------------------------------------------------------------------------
// One workgroup, PLAN_SUB threads per lane of the workers.  Bound by the round trips of its reads: calls of 128 to 512 sequences take 2 to 3 us more with it;
// without it every worker reads the whole batch.
constexpr int PLAN_SUB = 16, PLAN_THREADS = 64 * PLAN_SUB;
__device__ __forceinline__ int64_t sub_sum(int64_t x) {
#pragma unroll
  for (int i = 1; i < PLAN_SUB; i *= 2) x += __shfl_xor(x, i);
  return x;
}
template <bool MANY>
__global__ void __launch_bounds__(PLAN_THREADS) paged_plan_kernel(PagedArgs a, void* plan) {
  const int l = threadIdx.x / PLAN_SUB, sub = threadIdx.x % PLAN_SUB;
  if constexpr (!MANY) {
    Line<FEW_PAIRS> line;
    line.chunk = (a.batch + 63) >> 6;
    const int64_t sum = sub_sum(line.lane_sum(a, l, sub, PLAN_SUB));
    if (sub == 0) ((int64_t*)plan)[l] = sum;
  } else {
    __shared__ int64_t tiles[PLAN_THREADS / 64], keys[PLAN_THREADS / 64];
    __shared__ int longest[PLAN_THREADS / 64];
    Units<MANY_PAIRS> units;
    units.chunk = (a.batch + 63) >> 6;  // (> 1: what a lane keeps of its one sequence is not read)
    int64_t t, k;
    int most;
    units.lane_tiles(a, l, sub, PLAN_SUB, t, k, most);
    t = lane64(wave_scan64(t), 63);
    k = lane64(wave_scan64(k), 63);
    most = wave_max(most);
    const int wave = threadIdx.x >> 6;
    keys[wave] = k;  // (the same in all lanes)
    tiles[wave] = t;
    longest[wave] = most;
    __syncthreads();
    t = k = 0;
    most = 0;
    for (int w = 0; w < PLAN_THREADS / 64; ++w) {
      k += keys[w];
      t += tiles[w];
      most = longest[w] > most ? longest[w] : most;
    }
    units.lane_counts(a, l, sub, PLAN_SUB, 0, uniform64(t), uniform64(k), most);
    const int u = (int)sub_sum(units.lane_units), cu = (int)sub_sum(units.lane_cut_units), ct = (int)sub_sum(units.lane_cut_tiles);
    if (sub == 0) ((int4*)plan)[l] = make_int4(u, cu, ct, units.share);
  }
}

// ---- sum of the parts ------------------------------------------------------------------------------------------------------
// Workgroup w adds up the parts of the tile of record w, if there is one, in their order.  Threads: one per four elements of the tile, in
// blockIdx.y blocks, and where that leaves some over, runs of parts.
constexpr int REDUCE_THREADS = 256, REDUCE_SPLIT = 16;  // (many rows: workgroups per tile)
template <int QT, int DV>
__global__ void __launch_bounds__(REDUCE_THREADS) paged_reduce_kernel(PagedArgs a) {
  constexpr int RW = DV / 4;  // float4 of a row
  __shared__ float4 sums[REDUCE_THREADS];
  const CutTile t = a.cut[blockIdx.x];
  if (t.parts == 0) return;
  const int cols = t.pairs * RW, tid = threadIdx.x;
  const int groups = cols >= REDUCE_THREADS ? 1 : REDUCE_THREADS / cols;
  const int per = (t.parts + groups - 1) / groups;
  for (int c0 = blockIdx.y * REDUCE_THREADS; c0 < cols; c0 += gridDim.y * REDUCE_THREADS) {
    const int grp = groups > 1 ? tid / cols : 0, c = groups > 1 ? tid % cols : c0 + tid;
    const bool on = grp < groups && c < cols;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (on) {
      const int x1 = (grp + 1) * per < t.parts ? (grp + 1) * per : t.parts;
#pragma unroll 8
      for (int x = grp * per; x < x1; ++x) {
        const int64_t slot = x == 0 ? t.slot0 : t.next + (int64_t)(x - 1) * t.step;
        const float4 y = *(const float4*)(a.partial + slot * QT * DV + (int64_t)c * 4);
        s.x += y.x; s.y += y.y; s.z += y.z; s.w += y.w;
      }
    }
    if (groups > 1) {
      sums[tid] = s;
      __syncthreads();
      if (grp == 0 && on)
        for (int x = 1; x < groups; ++x) {
          const float4 y = sums[x * cols + c];
          s.x += y.x; s.y += y.y; s.z += y.z; s.w += y.w;
        }
    }
    if (on && grp == 0) {
      const int pair = t.pair0 + c / RW;
      const int64_t o = (int64_t)(t.row0 + pair / a.group) * a.heads + t.head * a.group + pair % a.group;
      store4(a, o * DV + (c % RW) * 4, s.x, s.y, s.z, s.w);
    }
  }
}

constexpr int TEAM = 8;
template <bool F32, int DQK, int DV, int NW, int AUX>
hipError_t launch_few(const PagedArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)a.grid), block(64 * NW);
  if (a.ts_w) hipLaunchKernelGGL((paged_few_kernel<F32, DQK, DV, true, NW, AUX>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((paged_few_kernel<F32, DQK, DV, false, NW, AUX>), grid, block, 0, stream, a);
  return hipGetLastError();
}
template <bool F32, int DQK, int DV>
hipError_t launch_few(const PagedArgs& a, hipStream_t stream) {
  if (a.whole == 2) return launch_few<F32, DQK, DV, TEAM, 0>(a, stream);
  return a.stream ? launch_few<F32, DQK, DV, 1, 2>(a, stream) : launch_few<F32, DQK, DV, 1, 0>(a, stream);
}
template <bool F32, int DQK>
hipError_t launch_few_dv(const PagedArgs& a, int d_v, hipStream_t stream) {
  return d_v == 32 ? launch_few<F32, DQK, 32>(a, stream)
                   : (d_v == 64 ? launch_few<F32, DQK, 64>(a, stream) : launch_few<F32, DQK, 128>(a, stream));
}
template <bool F32>
hipError_t launch_few_d(const PagedArgs& a, int d_qk, int d_v, hipStream_t stream) {
  return d_qk == 32 ? launch_few_dv<F32, 32>(a, d_v, stream)
                    : (d_qk == 64 ? launch_few_dv<F32, 64>(a, d_v, stream) : launch_few_dv<F32, 128>(a, d_v, stream));
}
template <int QT>
hipError_t launch_reduce(const PagedArgs& a, int d_v, hipStream_t stream) {
  const dim3 grid((unsigned)(QT > FEW_PAIRS ? a.records : a.workers), QT > FEW_PAIRS ? REDUCE_SPLIT : 1), block(REDUCE_THREADS);
  if (d_v == 32) hipLaunchKernelGGL((paged_reduce_kernel<QT, 32>), grid, block, 0, stream, a);
  else if (d_v == 64) hipLaunchKernelGGL((paged_reduce_kernel<QT, 64>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((paged_reduce_kernel<QT, 128>), grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_plan(const PagedArgs& a, int many, hipStream_t stream) {
  void* plan = const_cast<void*>(a.plan);
  if (many) hipLaunchKernelGGL((paged_plan_kernel<true>), dim3(1), dim3(PLAN_THREADS), 0, stream, a, plan);
  else hipLaunchKernelGGL((paged_plan_kernel<false>), dim3(1), dim3(PLAN_THREADS), 0, stream, a, plan);
  return hipGetLastError();
}

hipError_t launch_paged_few(const PagedArgs& a, int dtype_f32, int d_qk, int d_v, hipStream_t stream) {
  return dtype_f32 ? launch_few_d<true>(a, d_qk, d_v, stream) : launch_few_d<false>(a, d_qk, d_v, stream);
}

hipError_t launch_paged_reduce(const PagedArgs& a, int many, int d_v, hipStream_t stream) {
  return many ? launch_reduce<MANY_PAIRS>(a, d_v, stream) : launch_reduce<FEW_PAIRS>(a, d_v, stream);
}

}  // namespace hstu
