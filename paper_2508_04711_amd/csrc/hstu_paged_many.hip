// Attention of many new rows over a paged cache (bursts of events, hundreds of candidates against one history), bf16.
//
// With r (new row, query head) pairs per key/value head a row of the cache is worth r flops a byte: from about 128 on the
// matrix cores bound the pass and not the memory.  So a worker is a workgroup of four waves, 32 pairs each, which shares the tiles
// of 64 keys it streams through LDS, with the forward pass's layouts (hstu_mfma.h).  Tiles of
// 128 pairs are cut along the keys (Units, hstu_paged.h), so a call of two tiles fills the chip as one of hundreds does.
//   - A wave-wide copy fills rows of one group of 16, which lies inside one page: its buffer descriptor is the group's
//     rows, in scalar registers, and what lies behind the part's end or in a page that does not exist arrives as zeros.
//   - The tiles of keys that every pair sees go through the pipelined step without any mask; the last few, which the causal
//     diagonal crosses, through a loop that finishes a block at a time.
//   - P is rounded to bf16 once, as in the forward pass: outputs are off by 2.3e-3 of their norm, 1.7e-3 with the second term that few rows
//     keep.  That term is half as many matrix instructions again where these bound the pass (4 x 512..1024 new rows over
//     4096..16384, H = 8: 145 -> 188 us; 8 x 200..600 over 1024..8192, H = 4: 53 -> 65).
//   - Consecutive workers (the tiles of one head over one range of keys) run on one XCD and find each other's tiles in its L2.
#include "hstu_mfma.h"
#include "hstu_paged.h"

namespace hstu {

namespace {

constexpr int MANY_WAVES = 4;

// Descriptor of the rows [key, key + most) of one page, those before `end` and none of a page that does not exist.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t page_rsrc(const char* base, int64_t page_bytes, int row_bytes, const PagedView& c,
                                                            const PageIds& ids, int h, int key, int end, int most) {
  const int id = ids.get(key >> c.ps_log2);
  const int64_t at = ((int64_t)h << c.ps_log2) + (key & ((1 << c.ps_log2) - 1)), page = id < 0 ? 0 : id;
  return __builtin_amdgcn_make_buffer_rsrc((void*)(base + page * page_bytes + at * row_bytes), 0, rows_before(id, key, end, most) * row_bytes,
                                           0x00020000);
}

// Copies the wave's share of keys [key, key + 64) into an LDS tile (swizzled like tile_copy_async); rows from `end` on
// and rows without a page become zeros.  AUX 2: nontemporal (PagedArgs::stream).  base: K or V pages; ids holds the tile's entries.
template <int D, int AUX>
__device__ __forceinline__ void page_copy_async(char* tile, const char* base, int64_t page_bytes, const PagedView& c,
                                                const PageIds& ids, int h, int key, int end, int wave, int lane) {
  constexpr int RB = D * 2, CPR = D / 8, RPL = 64 / CPR, LOADS = ST / RPL;
  static_assert(RPL <= 16 && LOADS % MANY_WAVES == 0, "a copy stays inside 16 rows; every wave does as many");
  static_assert(MANY_WAVES * RPL % 16 == 0, "the lane's place in its 16 rows is the same in all of them");
  const int row = ((wave * RPL) & 15) + lane / CPR, voff = row * RB + (((lane % CPR) ^ swz<D>(row)) << 4);
  if (c.ps_log2 >= 6) {  // the tile is in one page (its first key is a multiple of 64): one descriptor for all of it
    const __amdgpu_buffer_rsrc_t rsrc = page_rsrc(base, page_bytes, RB, c, ids, h, key, end, ST);
    // (The group's offset in the vector register: the descriptor's bound is not defined for the scalar offset, and a
    // tile that ends inside the page, or has no page, has groups that lie behind it.)
    int group = voff + ((wave * RPL) & ~15) * RB;
    asm volatile("" : "+v"(group));  // (worked out at every copy: the loop has no registers for all groups' offsets)
#pragma unroll
    for (int i = 0; i < LOADS / MANY_WAVES; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, HSTU_LDS(void, tile + (i * MANY_WAVES + wave) * 1024), 16,
                                               group + i * MANY_WAVES * RPL * RB, 0, 0, AUX);
    return;
  }
#pragma unroll
  for (int i = 0; i < LOADS / MANY_WAVES; ++i) {
    const int idx = i * MANY_WAVES + wave;
    const __amdgpu_buffer_rsrc_t rsrc = page_rsrc(base, page_bytes, RB, c, ids, h, key + ((idx * RPL) & ~15), end, 16);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, HSTU_LDS(void, tile + idx * 1024), 16, voff, 0, 0, AUX);
  }
}

// The same for the timestamps of the 64 keys (one wave's work; a word per lane, 16 lanes per descriptor).
__device__ __forceinline__ void stamp_copy_async(int* tile, const PagedView& c, const PageIds& ids, int key, int end, int lane) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int k16 = key + 16 * i, id = ids.get(k16 >> c.ps_log2), rows = rows_before(id, k16, end, 16);
    const int32_t* p = c.ts + ((int64_t)(id < 0 ? 0 : id) << c.ps_log2) + (k16 & ((1 << c.ps_log2) - 1));
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, rows * 4, 0x00020000);
    if (lane >> 4 == i) __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, HSTU_LDS(void, tile), 4, (lane & 15) * 4, 0, 0, 0);
  }
}

// Scores start from the bias of the lane's pair and the block's keys, or from zero.
template <bool BIAS>
struct PagedInit {
  const int* ts;      // timestamps of the block's keys (LDS)
  const float* wtab;
  int tq, nb, f, hh;
  __device__ __forceinline__ void operator()(f32x16& s) const {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      if constexpr (BIAS) s[r] = wtab[bias_bucket(abs_diff(tq, ts[8 * (r >> 2) + 4 * hh + (r & 3)]), nb, f)];
      else s[r] = 0.f;
    }
  }
};

// One step of the pipeline over blocks of 32 keys: the matrix instructions of S(i + 1) = K(i + 1) Q^T and of O^T += V(i - 1)^T P(i - 1)^T,
// and between them the SiLU of block i.  A wave issues one instruction at a time and waits where one needs the last
// one's result, so the five instructions of an element's SiLU are spread over as many slots: what stands in a slot belongs to different
// elements.  (4 x 512..1024 new rows over 4096..16384, H = 8: 148 us with an element's five instructions in one slot, 144 so.)  The empty
// asm statements keep the compiler from moving the vector instructions behind the matrix instructions (166 us).
template <int DQK, int DV, bool PV, class Init>
__device__ __forceinline__ void many_step(const Init& init, const char* kn, int bn, const char* vp, int bp,
                                          const RowAddr<DQK>& ra, const ColAddr<DV>& ca, const bf16x8 (&qreg)[DQK / 16],
                                          const f32x16& s_in, f32x16& s_out, const bf16x8 (&p_prev)[2], bf16x8 (&p_cur)[2],
                                          f32x16 (&oacc)[DV / 32], float c1) {
  constexpr int KS = DQK / 16, NPV = DV / 16, NSL = KS > NPV ? KS : NPV;
  constexpr int SLOTS = 2 * NSL, E = (16 + SLOTS - 1) / SLOTS;  // elements that enter per slot
  constexpr int AHEAD = 3;  // operand reads in flight ahead of their use
  bf16x8 ka[KS], va[NPV];
  float x[16];
  auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
  auto scale = [&](int h) {
#pragma unroll
    for (int i = h * E; i < (h + 1) * E && i < 16; ++i) x[i] = s_in[i] * c1;
  };
  auto silu = [&](int h) {  // slot h: elements of slots h, h - 1, h - 2, h - 3 one instruction further each
#pragma unroll
    for (int i = h * E; i < (h + 1) * E && i < 16; ++i) {
      x[i] = __builtin_amdgcn_exp2f(x[i]);
      asm volatile("" : "+v"(x[i]));
    }
    scale(h + 1);
    if (h >= 1)
#pragma unroll
      for (int i = (h - 1) * E; i < h * E && i < 16; ++i) x[i] = 1.0f + x[i];
    if (h >= 2)
#pragma unroll
      for (int i = (h - 2) * E; i < (h - 1) * E && i < 16; ++i) {
        x[i] = __builtin_amdgcn_rcpf(x[i]);
        asm volatile("" : "+v"(x[i]));
      }
    if (h >= 3)
#pragma unroll
      for (int i = (h - 3) * E; i < (h - 2) * E && i < 16; ++i) x[i] = s_in[i] * x[i];
  };
  init(s_out);
#pragma unroll
  for (int m = 0; m < AHEAD; ++m) {
    if (m < KS) ka[m] = ra.read(kn, bn, m);
    if (PV && m < NPV) va[m] = ca.read(vp, bp * 2 + (m & 1), m >> 1);
  }
  scale(0);
  fence();
#pragma unroll
  for (int m = 0; m < NSL; ++m) {
    if (m < KS) s_out = mfma(ka[m], qreg[m], s_out);
    if (m + AHEAD < KS) ka[m + AHEAD] = ra.read(kn, bn, m + AHEAD);
    silu(2 * m);
    fence();
    if (PV && m < NPV) oacc[m >> 1] = mfma(va[m], p_prev[m & 1], oacc[m >> 1]);
    if (PV && m + AHEAD < NPV) va[m + AHEAD] = ca.read(vp, bp * 2 + ((m + AHEAD) & 1), (m + AHEAD) >> 1);
    silu(2 * m + 1);
    fence();
  }
#pragma unroll
  for (int h = SLOTS; h < SLOTS + 3; ++h) silu(h);
  p_cur[0] = pack8(x);
  p_cur[1] = pack8(x + 8);
  fence();
}

template <int DQK, int DV, bool BIAS, int AUX>
__global__ void __launch_bounds__(MANY_WAVES * 64, 2) paged_many_kernel(PagedArgs a) {
  constexpr int KB = ST * DQK * 2, VB = ST * DV * 2;
  // two buffers each, apart from each other, copies one tile ahead (see hstu_fwd_bf16)
  __shared__ __attribute__((aligned(1024))) char kmem0[KB];
  __shared__ __attribute__((aligned(1024))) char kmem1[KB];
  __shared__ __attribute__((aligned(1024))) char vmem0[VB];
  __shared__ __attribute__((aligned(1024))) char vmem1[VB];
  __shared__ __attribute__((aligned(1024))) int tmem0[BIAS ? ST : 1];
  __shared__ __attribute__((aligned(1024))) int tmem1[BIAS ? ST : 1];
  __shared__ float wtab[BIAS ? MAX_TS_BUCKETS : 1];
  auto kbuf = [&](int b) { return b ? kmem1 : kmem0; };
  auto vbuf = [&](int b) { return b ? vmem1 : vmem0; };
  auto tbuf = [&](int b) { return b ? tmem1 : tmem0; };

  const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Units<MANY_PAIRS> units;
  units.init(a);
  if (blockIdx.x == 0)  // (records that no tile uses)
    for (int x = units.total_cut + tid; x < a.records; x += MANY_WAVES * 64) a.cut[x].parts = 0;
  const int64_t w = worker_place(blockIdx.x, units.total);
  if (w >= units.total) return;
  if constexpr (BIAS)
    for (int x = tid; x < a.nb; x += MANY_WAVES * 64) wtab[x] = a.ts_w[x];
  const ManyUnit sg = units.find(a, uniform32((int)w));
  if (sg.cut >= 0 && sg.piece == 0 && tid == 0) {
    CutTile c = {};
    c.parts = sg.parts > 1 ? sg.parts : 0;
    c.pairs = sg.pairs; c.pair0 = sg.t * MANY_PAIRS; c.head = sg.h; c.row0 = sg.row0;
    c.slot0 = sg.slot; c.next = sg.slot + sg.tiles; c.step = sg.tiles;
    a.cut[sg.cut] = c;
  }
  if (sg.piece >= sg.parts) return;  // (keys that no row of the tile sees)

  RowAddr<DQK> ra;
  ColAddr<DV> ca;
  ra.init(n, hh);
  ca.init(lane);
  const float c1 = -a.alpha * 1.4426950408889634f;
  const int slot = wave * 32 + n;  // the lane's pair in the tile
  const int pair = sg.t * MANY_PAIRS + slot, row = pair / a.group, head = sg.h * a.group + pair % a.group;
  const bool on = slot < sg.pairs, wave_on = wave * 32 < sg.pairs;
  const int64_t qrow = sg.row0 + row;
  bf16x8 qreg[DQK / 16];
#pragma unroll
  for (int s = 0; s < DQK / 16; ++s) {
    u32x4 z = {0, 0, 0, 0};
    if (on) z = *(const u32x4*)(a.q + qrow * a.q_stride + (int64_t)head * DQK * 2 + s * 32 + hh * 16);
    qreg[s] = __builtin_bit_cast(bf16x8, z);
  }
  int tq = 0;
  if constexpr (BIAS) tq = on ? a.ts_q[qrow] : 0;
  f32x16 oacc[DV / 32];
#pragma unroll
  for (int i = 0; i < DV / 32; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[i][r] = 0.f;

  // Tiles of keys: T in all, of which every pair sees all keys of the first T0.
  const int T = (sg.k1 - sg.k0 + ST - 1) / ST;
  const int T0 = sg.lim0 >= sg.k1 ? T : (sg.lim0 > sg.k0 ? (sg.lim0 - sg.k0) / ST : 0);
  PageIds ids;
  const int entries = (sg.k1 + (1 << a.c.ps_log2) - 1) >> a.c.ps_log2;
  auto copy_k = [&](int t, int buf) __attribute__((always_inline)) {
    const int key = sg.k0 + t * ST, last = key + ST - 1 < sg.k1 ? key + ST - 1 : sg.k1 - 1;
    // (V's copies are up to a tile behind K's: a refill starts there)
    if (!ids.holds(last >> a.c.ps_log2)) ids.fill(a.c, sg.b, (key - ST > sg.k0 ? key - ST : sg.k0) >> a.c.ps_log2, entries);
    page_copy_async<DQK, AUX>(kbuf(buf), a.c.k, a.c.k_page, a.c, ids, sg.h, key, sg.k1, wave, lane);
    if constexpr (BIAS)
      if (wave == 0) stamp_copy_async(tbuf(buf), a.c, ids, key, sg.k1, lane);
  };
  auto copy_v = [&](int t, int buf) __attribute__((always_inline)) {
    page_copy_async<DV, AUX>(vbuf(buf), a.c.v, a.c.v_page, a.c, ids, sg.h, sg.k0 + t * ST, sg.k1, wave, lane);
  };
  auto init_of = [&](int buf, int blk) __attribute__((always_inline)) {
    return PagedInit<BIAS>{tbuf(buf) + blk * 32, wtab, tq, a.nb, a.f, hh};
  };

  if (T > 0) {
    ids.fill(a.c, sg.b, sg.k0 >> a.c.ps_log2, entries);
    copy_k(0, 0);
    copy_v(0, 0);
    if (T > 1 && T0 > 0) copy_k(1, 1);
  }
  tile_copy_wait<0>();
  if constexpr (BIAS) __syncthreads();  // (the table)
  tile_barrier();

  // The pipelined loop (see hstu_fwd_bf16): iteration j does the steps 2j+1 and 2j+2, step i S(i+1), P(i) and P(i-1) V(i-1).
  if (T0 > 0) {
    f32x16 sacc[2];   // S of the blocks of even / odd index
    bf16x8 pb[2][2];  // P (two 16-key halves) of the blocks of even / odd index
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int r = 0; r < 16; ++r) sacc[x][r] = 0.f;
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int e = 0; e < 8; ++e) pb[x][y][e] = (__bf16)0.f;
    }
    if (wave_on) {
      init_of(0, 0)(sacc[0]);
#pragma unroll
      for (int ks = 0; ks < DQK / 16; ++ks) sacc[0] = mfma(ra.read(kbuf(0), 0, ks), qreg[ks], sacc[0]);
      many_step<DQK, DV, false>(init_of(0, 1), kbuf(0), 1, vbuf(0), 0, ra, ca, qreg, sacc[0], sacc[1], pb[1], pb[0], oacc,
                               c1);
    }
    tile_barrier();
    auto iter = [&](int j, auto buf_tag) __attribute__((always_inline)) {
      constexpr int B0 = decltype(buf_tag)::value, B1 = B0 ^ 1;
      if (j + 2 <= T0 && j + 2 < T) copy_k(j + 2, B0);
      if (j + 1 < T) copy_v(j + 1, B1);
      if (wave_on) {
        many_step<DQK, DV, true>(init_of(B1, 0), kbuf(B1), 0, vbuf(B0), 0, ra, ca, qreg, sacc[1], sacc[0], pb[0], pb[1], oacc,
                                c1);
        if (j + 1 < T0)
          many_step<DQK, DV, true>(init_of(B1, 1), kbuf(B1), 1, vbuf(B0), 1, ra, ca, qreg, sacc[0], sacc[1], pb[1], pb[0],
                                  oacc, c1);
      }
      tile_copy_wait<0>();
      tile_barrier();
    };
    for (int j = 0; j < T0; j += 2) {
      iter(j, std::integral_constant<int, 0>{});
      if (j + 1 < T0) iter(j + 1, std::integral_constant<int, 1>{});
    }
    if (wave_on) {  // P V of the last block
      const char* vt = vbuf((T0 - 1) & 1);
#pragma unroll
      for (int c = 0; c < DV / 32; ++c) {
        oacc[c] = mfma(ca.read(vt, 2, c), pb[1][0], oacc[c]);
        oacc[c] = mfma(ca.read(vt, 3, c), pb[1][1], oacc[c]);
      }
    }
    tile_barrier();  // (the next copies go where these values were read)
  }

  // Tiles that the diagonal crosses, a block at a time (one or two per tile of pairs: the copies are waited for, in
  // exchange for a single loop over both buffers).  Tile t's K and V are in the buffers t % 2.
  // Keys that the lane's pair and the wave's last pair see:
  int lim = sg.n, lim1 = sg.n;
  if (a.causal) {
    const int p0 = sg.t * MANY_PAIRS + wave * 32, most = sg.pairs - wave * 32;
    const int64_t past = (int64_t)sg.n - sg.m + 1;
    lim = clampi(past + row, 0, sg.n);
    lim1 = uniform32(clampi(past + (p0 + (most > 32 ? 32 : (most > 1 ? most : 1)) - 1) / a.group, 0, sg.n));
  }
  for (int t = T0; t < T; ++t) {
    const int B = t & 1;
    int hl = hh;
    asm volatile("" : "+v"(hl));  // (as above)
    if (t + 1 < T) {
      copy_k(t + 1, B ^ 1);
      copy_v(t + 1, B ^ 1);
    }
#pragma unroll 1
    for (int blk = 0; blk < 2; ++blk) {
      const int key = sg.k0 + t * ST + blk * 32;
      if (!wave_on || key >= lim1 || key >= sg.k1) break;
      f32x16 s;
      init_of(B, blk)(s);
#pragma unroll
      for (int ks = 0; ks < DQK / 16; ++ks) {
        s = mfma(ra.read(kbuf(B), blk, ks), qreg[ks], s);
        if (ks & 1) __builtin_amdgcn_sched_barrier(0);  // (few registers are left)
      }
      float p[16];
      const VisBefore vis(lim - 1 - key, hl);
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = vis(r) ? s[r] * sigmoid_scaled(s[r], c1) : 0.f;
      bf16x8 p0 = pack8(p), p1 = pack8(p + 8);
      // Rows of V that some pairs of the wave see and others do not: an infinity or NaN there times a zero of P would reach
      // the pairs that do not see it.  So the product takes the rows before the first such one alone ...
      int first = 32;  // (rows of the block; a lane's operand holds four runs of four of them)
#pragma unroll
      for (int y = 1; y >= 0; --y) {
        uint32_t lo = 0, hi = 0;  // exponents of all ones in rows 16 y + 4 hl + 0..3 and in rows 16 y + 8 + 4 hl + 0..3
#pragma unroll
        for (int c = 0; c < DV / 32; ++c) {
          const u32x4 v = __builtin_bit_cast(u32x4, ca.read(vbuf(B), blk * 2 + y, c));
          const uint32_t w[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t bits = (uint32_t)((w[e] & 0x7f80u) == 0x7f80u) | (uint32_t)((w[e] & 0x7f800000u) == 0x7f800000u) << 1;
            if (e < 2) lo |= bits << (2 * e); else hi |= bits << (2 * e - 4);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        const int at_hi = hi ? 16 * y + 8 + 4 * hl + __builtin_ctz(hi) : 32, at_lo = lo ? 16 * y + 4 * hl + __builtin_ctz(lo) : 32;
        first = at_hi < first ? at_hi : first;
        first = at_lo < first ? at_lo : first;
      }
      first = wave_min(first);
      uint32_t keep[8];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int rows = first - 8 * x - 4 * hl, c = rows < 0 ? 0 : (rows < 4 ? rows : 4);
        keep[2 * x] = c >= 2 ? ~0u : (c == 1 ? 0xffffu : 0u);
        keep[2 * x + 1] = c >= 4 ? ~0u : (c == 3 ? 0xffffu : 0u);
      }
      // (both factors of the rows that are left out: theirs may be infinite too)
      u32x4 w0 = __builtin_bit_cast(u32x4, p0), w1 = __builtin_bit_cast(u32x4, p1);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w0[e] &= keep[e];
        w1[e] &= keep[4 + e];
      }
      p0 = __builtin_bit_cast(bf16x8, w0);
      p1 = __builtin_bit_cast(bf16x8, w1);
#pragma unroll
      for (int c = 0; c < DV / 32; ++c)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          u32x4 v = __builtin_bit_cast(u32x4, ca.read(vbuf(B), blk * 2 + y, c));
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] &= keep[4 * y + e];
          oacc[c] = mfma(__builtin_bit_cast(bf16x8, v), y ? p1 : p0, oacc[c]);
          if (y) __builtin_amdgcn_sched_barrier(0);
        }
      // ... and the others are added pair by pair where they are seen.
#pragma unroll 1
      for (int k = first; k < 32; ++k) {
        float dot = 0.f;
#pragma unroll
        for (int ks = 0; ks < DQK / 16; ++ks) {
          const bf16x8 x = *HSTU_LDS(bf16x8, kbuf(B) + lds_off<DQK>(blk * 32 + k, ks * 2 + hl));
          u32x4 qw = __builtin_bit_cast(u32x4, qreg[ks]);
          asm volatile("" : "+v"(qw));  // (converted here, not once for the loop: no registers for that)
          const bf16x8 y = __builtin_bit_cast(bf16x8, qw);
#pragma unroll
          for (int e = 0; e < 8; ++e) dot = __builtin_fmaf((float)x[e], (float)y[e], dot);
          __builtin_amdgcn_sched_barrier(0);
        }
        dot += __shfl_xor(dot, 32);
        if constexpr (BIAS) dot += wtab[bias_bucket(abs_diff(tq, tbuf(B)[blk * 32 + k]), a.nb, a.f)];
        if (key + k < lim) {
          const float x = (float)(__bf16)(dot * sigmoid_scaled(dot, c1));
#pragma unroll
          for (int c = 0; c < DV / 32; ++c)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
              const bf16x4 v = *HSTU_LDS(bf16x4, vbuf(B) + lds_off<DV>(blk * 32 + k, c * 4 + q4) + 8 * hl);
#pragma unroll
              for (int e = 0; e < 4; ++e) oacc[c][4 * q4 + e] = __builtin_fmaf(x, (float)v[e], oacc[c][4 * q4 + e]);
              __builtin_amdgcn_sched_barrier(0);
            }
        }
      }
    }
    tile_copy_wait<0>();
    tile_barrier();
  }

  if (on) {
    if (sg.parts == 1)
      store_owner_major<DV>(a.o, (qrow * a.heads + head) * DV, oacc, a.alpha * a.inv_n, hh, 0, a.out_f32);
    else
      store_owner_major<DV>(a.partial, ((int64_t)sg.slot * MANY_PAIRS + slot) * DV, oacc, 1.f, hh, 0, 1);
  }
}

template <int DQK, int DV, int AUX>
hipError_t launch_many(const PagedArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)a.grid), block(MANY_WAVES * 64);
  if (a.ts_w) hipLaunchKernelGGL((paged_many_kernel<DQK, DV, true, AUX>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((paged_many_kernel<DQK, DV, false, AUX>), grid, block, 0, stream, a);
  return hipGetLastError();
}
template <int DQK, int DV>
hipError_t launch_many(const PagedArgs& a, hipStream_t stream) {
  return a.stream ? launch_many<DQK, DV, 2>(a, stream) : launch_many<DQK, DV, 0>(a, stream);
}
template <int DQK>
hipError_t launch_many_dv(const PagedArgs& a, int d_v, hipStream_t stream) {
  return d_v == 32 ? launch_many<DQK, 32>(a, stream) : (d_v == 64 ? launch_many<DQK, 64>(a, stream) : launch_many<DQK, 128>(a, stream));
}

}  // namespace

hipError_t launch_paged_many(const PagedArgs& a, int d_qk, int d_v, hipStream_t stream) {
  return d_qk == 32 ? launch_many_dv<32>(a, d_v, stream)
                    : (d_qk == 64 ? launch_many_dv<64>(a, d_v, stream) : launch_many_dv<128>(a, d_v, stream));
}

}  // namespace hstu
