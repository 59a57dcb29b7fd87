// What the kernels of the paged cache share (not part of the C ABI): the view of a cache, and the schedule of the attention of
// new rows over it.
#pragma once
#include "hstu_common.h"

namespace hstu {

// Rows of a sequence that count at most (loops add up to a few thousand to a key's number).
constexpr int32_t MAX_KEYS = 0x7fff0000;

// A paged cache on the device.  Page p holds, per key/value head, `ps` rows: [heads][ps][d].
struct PagedView {
  const char* k;              // pages of K and V
  const char* v;
  int64_t k_page, v_page;     // bytes from page to page
  const int32_t* table;       // [batch][table_stride] page ids
  int64_t table_stride;
  const int32_t* lens;        // [batch] rows in the cache, the new ones among them
  int32_t* ts;                // [num_pages][ps] timestamps, or null
  uint32_t num_pages;
  int32_t ps_log2;            // page size 16 << n
  int32_t cap;                // rows a sequence's part of the table has room for
};

struct CutTile;
struct PagedArgs {
  PagedView c;
  const char* q;              // [rows][heads][d_qk], rows q_stride bytes apart
  int64_t q_stride;
  const int32_t* off;         // [batch + 1] offsets of the new rows
  const int32_t* ts_q;        // timestamps of the new rows; ts_w: the bias table (nb entries, 2^f groups an octave)
  const float* ts_w;
  int32_t nb, f;
  void* o;                    // [rows][heads][d_v]
  const void* plan;           // large batches: the lanes' sums of Line or Units (paged_plan_kernel), or null
  CutTile* cut;               // records of cut tiles, one per worker
  float* partial;             // partial results, two per worker
  int32_t batch, rows, heads, kv_heads, group;
  int32_t causal, out_f32;
  float alpha, inv_n;
  int32_t workers;            // a multiple of 8; many rows: the workgroups that run at once
  int32_t records;            // many rows: records of cut tiles that there is room for
  int32_t grid;               // workgroups: enough for all workers; many rows: for all tiles and twice the workers
  int32_t whole;              // 1: every worker takes one tile, uncut; 2: ... and is a team of waves
  int32_t min_share;          // keys a worker takes at least
  int32_t stream;             // the cached rows are more than the memory-side cache would keep: loads that allocate nothing there
};

// The schedule.  For one key/value head of one sequence the (new row, query head) pairs that read it are numbered
// row * group + head and cut into tiles of QT pairs; a tile streams over the keys that its last row sees.  What a tile costs is
// counted in keys times `group` (so that the causal sum over tiles has a closed form), TILE_KEYS for its own loads and stores
// included.  The tiles of all sequences and heads in order form one line, of which every worker takes an equal length
// (min_share at least): no sequence however long or short leaves a worker idle, and nothing is read on the host.  A worker that
// starts or ends inside a tile writes an fp32 partial result; SiLU attention is a plain sum over keys, so joining the parts is
// an addition (reduce kernel, in the order of the keys: results repeat bit for bit).
constexpr int TILE_KEYS = 32;

struct SeqWork {
  int m, n;      // new rows, cached rows
  int row0;      // first new row
  int tiles;     // of one head
  int64_t base;  // cost of tile t is base + (causal ? (t + 1) * QT : 0)
  int64_t cost;  // of one head
};

__device__ __forceinline__ int64_t tiles_cost(const SeqWork& s, int64_t t, int qt, bool causal) {
  return t * s.base + (causal ? qt * (t * (t + 1) / 2) : 0);
}

template <int QT>
__device__ __forceinline__ SeqWork seq_work(const PagedArgs& a, int m, int n, int row0) {
  SeqWork s;
  s.m = m; s.n = n; s.row0 = row0;
  s.tiles = (int)(((int64_t)m * a.group + QT - 1) / QT);
  if (a.whole) {
    s.base = 1;
    s.cost = s.tiles;
  } else {
    const int keys = a.causal ? (n > m ? n - m : 0) : n;
    s.base = (int64_t)(keys + TILE_KEYS) * a.group;
    s.cost = tiles_cost(s, s.tiles, QT, a.causal != 0);
  }
  return s;
}
template <int QT>
__device__ __forceinline__ SeqWork read_work(const PagedArgs& a, int b) {
  int r, e;
  seq_range(a.off, b, a.rows, r, e);
  return seq_work<QT>(a, e - r, clampi(a.c.lens[b], 0, a.c.cap), r);
}

// Place of cost unit x: sequence, head, tile, and the unit's place inside the tile.
struct Place {
  int b, h, t;
  int64_t u;     // place inside the tile
  SeqWork s;
};

__device__ __forceinline__ int64_t join64(uint32_t lo, uint32_t hi) { return (int64_t)(((uint64_t)hi << 32) | lo); }
__device__ __forceinline__ int64_t uniform64(int64_t x) {
  return join64(__builtin_amdgcn_readfirstlane((int)(uint32_t)x), __builtin_amdgcn_readfirstlane((int)(x >> 32)));
}
__device__ __forceinline__ int64_t lane64(int64_t x, int l) {
  return join64(__builtin_amdgcn_readlane((int)(uint32_t)x, l), __builtin_amdgcn_readlane((int)(x >> 32), l));
}
__device__ __forceinline__ int uniform32(int x) { return __builtin_amdgcn_readfirstlane(x); }
// What the compiler cannot see to be the same in all lanes it keeps in vector registers, and loops over the lanes to make a
// buffer descriptor of it.
__device__ __forceinline__ Place uniform_place(const Place& p) {
  Place r;
  r.b = uniform32(p.b); r.h = uniform32(p.h); r.t = uniform32(p.t);
  r.u = uniform64(p.u);
  r.s.m = uniform32(p.s.m); r.s.n = uniform32(p.s.n); r.s.row0 = uniform32(p.s.row0); r.s.tiles = uniform32(p.s.tiles);
  r.s.base = uniform64(p.s.base); r.s.cost = uniform64(p.s.cost);
  return r;
}
// Inclusive prefix sums of 64-bit values over the wave, on the vector pipe.
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t dpp64(int64_t x) {
  return join64(__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xf, false),
                __builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ int64_t wave_scan64(int64_t x) {
  x += dpp64<0x111, 0xf>(x);  // row_shr:1, 2, 4, 8
  x += dpp64<0x112, 0xf>(x);
  x += dpp64<0x114, 0xf>(x);
  x += dpp64<0x118, 0xf>(x);
  x += dpp64<0x142, 0xa>(x);  // row_bcast:15 into rows 1 and 3, row_bcast:31 into rows 2 and 3
  x += dpp64<0x143, 0xc>(x);
  return x;
}
// y / c of non-negative numbers (uniform): almost always both have 32 bits, where a division is much shorter.
__device__ __forceinline__ int64_t quotient(int64_t y, int64_t c) {
  if ((uint64_t)(y | c) >> 32 == 0) return (uint32_t)y / (uint32_t)c;
  return y / c;
}

// The line of all work, seen by one wave: lane i sums the sequences [i * chunk, (i + 1) * chunk).
template <int QT>
struct Line {
  int chunk;
  int64_t incl, sum;  // of the lane's sequences and all before them; of the lane's alone
  int64_t total;
  int m, n, row0;     // chunk 1: the lane's sequence

  __device__ __forceinline__ void init(const PagedArgs& a) {
    const int lane = threadIdx.x & 63;
    chunk = (a.batch + 63) >> 6;
    m = n = row0 = 0;
    sum = a.plan ? ((const int64_t*)a.plan)[lane] : lane_sum(a, lane, 0, 1);
    incl = wave_scan64(sum);
    total = lane64(incl, 63);
  }

  // The cost of every `step`-th sequence of lane l's from i0 on.  Of a large batch a kernel of one workgroup sums it up, once for
  // all workers; of a smaller one every worker does, which saves a launch.
  __device__ __forceinline__ int64_t lane_sum(const PagedArgs& a, int l, int i0, int step) {
    const int64_t b0 = (int64_t)l * chunk;
    int64_t x = 0;
    // (no branch on the sequence: the loads of several are in flight together)
#pragma unroll 4
    for (int i = i0; i < chunk; i += step) {
      const bool in = b0 + i < a.batch;
      const SeqWork s = read_work<QT>(a, in ? (int)b0 + i : a.batch - 1);
      x += in ? s.cost : 0;
      m = s.m; n = s.n; row0 = s.row0;
    }
    return x * a.kv_heads;
  }

  // The work of sequence b (uniform): from the lane that has read it already where every lane has one.
  __device__ __forceinline__ SeqWork work(const PagedArgs& a, int b) const {
    if (chunk > 1) return read_work<QT>(a, b);
    return seq_work<QT>(a, __builtin_amdgcn_readlane(m, b), __builtin_amdgcn_readlane(n, b),
                        __builtin_amdgcn_readlane(row0, b));
  }

  // (x < total)
  __device__ __forceinline__ Place find(const PagedArgs& a, int64_t x) const {
    return uniform_place(find_place(a, x));
  }
  __device__ __forceinline__ Place find_place(const PagedArgs& a, int64_t x) const {
    const int lane = threadIdx.x & 63;
    const uint64_t past = __ballot(incl <= x);
    const int l = __popcll(past);  // first lane whose sum reaches beyond x
    int64_t before = lane64(incl - sum, l);
    int b = l * chunk;
    for (int left = chunk; chunk > 1 && left > 0; left -= 64) {  // sequences b .. b + 63 of the lane's, one per lane
      int64_t c = 0;
      if (lane < left && b + lane < a.batch) c = read_work<QT>(a, b + lane).cost * a.kv_heads;
      const int64_t in = wave_scan64(c);
      const uint64_t p = __ballot(before + in <= x);
      const int j = __popcll(p);
      if (j < 64) {
        before += lane64(in - c, j);
        b += j;
        break;
      }
      before += lane64(in, 63);
      b += 64;
    }
    Place r;
    r.b = __builtin_amdgcn_readfirstlane(b);
    r.s = work(a, r.b);
    r.h = 0;
    r.t = 0;
    int64_t y = uniform64(x - before);
    if (a.kv_heads > 1) {
      r.h = (int)quotient(y, r.s.cost);
      y -= (int64_t)r.h * r.s.cost;
    }
    if (r.s.tiles > 1) {
      const bool causal = a.causal && !a.whole;
      if (!causal) {
        r.t = (int)quotient(y, r.s.base);
      } else {
        int lo = 0, hi = r.s.tiles;  // tiles_cost(lo) <= y < tiles_cost(hi)
        while (hi - lo > 1) {
          const int mid = lo + (hi - lo) / 2;
          if (tiles_cost(r.s, mid, QT, true) <= y) lo = mid; else hi = mid;
        }
        r.t = lo;
      }
      y -= tiles_cost(r.s, r.t, QT, causal);
    }
    r.u = y;
    return r;
  }

  // Moves on to the next tile of the line.
  __device__ __forceinline__ void next(const PagedArgs& a, Place& p) const {
    next_place(a, p);
    p = uniform_place(p);
  }
  __device__ __forceinline__ void next_place(const PagedArgs& a, Place& p) const {
    p.u = 0;
    if (++p.t < p.s.tiles) return;
    p.t = 0;
    if (++p.h < a.kv_heads) return;
    p.h = 0;
    do {
      if (++p.b >= a.batch) return;
      p.s = work(a, p.b);
    } while (p.s.cost == 0);
  }
};

// The length of the line a worker takes, and the workers that get any.
__device__ __forceinline__ int64_t share_of(const PagedArgs& a, int64_t total) {
  if (a.whole) return 1;
  const int64_t s = quotient(total + a.workers - 1, a.workers), least = (int64_t)a.min_share * a.group;
  return uniform64(s > least ? s : least);
}

// Workers in the order of the line: consecutive ones, which may share keys (tiles of one head, one range), are put on one XCD.
// Workgroups are dealt to the 8 XCDs in turn.  (A permutation of the workers.)
__device__ __forceinline__ int64_t worker_place(int w, int64_t active) {
  const int64_t per = (active + 7) >> 3;
  return w < 8 * per ? (int64_t)(w & 7) * per + (w >> 3) : w;
}

// What the reduce kernel has to know of a cut tile: its parts are in slots slot0 and next, next + step, ...  Few rows: every worker
// writes a record, of the tile that it began and did not finish.
struct CutTile {
  int32_t parts;   // or 0: no such tile
  int32_t pairs, pair0, head, row0;
  int32_t slot0, next, step;
};

// One tile's part [u0, u1) of its cost, as keys [k0, k1).
struct Segment {
  int64_t u0, u1, cost;
  int k0, k1;    // keys of this part
  int lim0;      // keys the tile's first row sees
  int vis;       // keys its last row sees
  int pairs;     // pairs in the tile
  bool first, last;  // the part holds the tile's first / last keys
};

template <int QT>
__device__ __forceinline__ Segment make_segment(const PagedArgs& a, const SeqWork& s, int t, int64_t u0, int64_t room) {
  Segment g;
  const bool causal = a.causal && !a.whole;
  g.cost = s.base + (causal ? (int64_t)(t + 1) * QT : 0);
  g.u0 = u0;
  g.u1 = g.cost - u0 < room ? g.cost : u0 + room;
  g.first = u0 == 0;
  g.last = g.u1 == g.cost;
  const int64_t all = (int64_t)s.m * a.group, p0 = (int64_t)t * QT;
  g.pairs = all - p0 < QT ? (int)(all - p0) : QT;
  g.vis = s.n;
  g.lim0 = s.n;
  if (a.causal) {
    const int row0 = (int)(p0 / a.group), row1 = (int)((p0 + g.pairs - 1) / a.group);
    g.lim0 = clampi((int64_t)s.n - s.m + row0 + 1, 0, s.n);
    g.vis = clampi((int64_t)s.n - s.m + row1 + 1, 0, s.n);
  }
  // (cuts lie at multiples of 32 keys; the part after a cut works the same key out)
  auto key = [&](int64_t u) {
    const int64_t k = (quotient(u, a.group) - TILE_KEYS) & ~(int64_t)31;
    return clampi(k, 0, g.vis);
  };
  g.k0 = uniform32(g.first ? 0 : key(g.u0));
  g.k1 = uniform32(g.last ? g.vis : key(g.u1));
  g.lim0 = uniform32(g.lim0);
  g.vis = uniform32(g.vis);
  g.pairs = uniform32(g.pairs);
  g.u1 = uniform64(g.u1);
  return g;
}

// ---- the schedule of calls of many rows ----------------------------------------------------------------------------------
// There the tiles of one head read the same keys several times over: workers that run side by side stream the same keys at the same
// time, and all but the first find them in their XCD's L2.  So all tiles of a head are cut at the same keys, into C pieces each
// (C: its sequence's length over a common share), units are ordered sequence, head, piece, tile, and every workgroup takes one
// unit.  More units than run at once would be a second round of the chip for a few of them, and more partial results, of 64 KB
// each at d_v = 128: see find_share.
struct ManyUnit {
  int b, m, n, row0, tiles;
  int h, t;
  int k0, k1;      // keys of the unit, k1 <= vis
  int lim0, vis;   // keys that the tile's first and last row see
  int pairs;
  int parts;       // pieces of this tile that see any keys (1: uncut)
  int piece;
  int slot, cut;   // where the sequence's tiles are cut: the unit's slot, the tile's record (else -1)
};

template <int QT>
struct Units {
  int chunk, share;
  int m, n, row0;                    // chunk 1: the lane's sequence
  int units, cut_units, cut_tiles;   // of the lane's sequences and all before them
  int lane_units, lane_cut_units, lane_cut_tiles;
  int total, total_cut;

  struct Counts { int pieces, units, cut_units, cut_tiles; };
  __device__ __forceinline__ Counts counts(const PagedArgs& a, int m_, int n_) const {
    const int tiles = (int)(((int64_t)m_ * a.group + QT - 1) / QT);
    Counts c;
    c.pieces = !a.whole && n_ > share ? (int)(((int64_t)n_ + share - 1) / share) : 1;
    c.units = tiles * c.pieces * a.kv_heads;
    c.cut_units = c.pieces > 1 ? c.units : 0;
    c.cut_tiles = c.pieces > 1 ? tiles * a.kv_heads : 0;
    return c;
  }
  __device__ __forceinline__ void read(const PagedArgs& a, int b, int& m_, int& n_, int& r) const {
    int e;
    seq_range(a.off, b, a.rows, r, e);
    m_ = e - r;
    n_ = clampi(a.c.lens[b], 0, a.c.cap);
  }

  __device__ __forceinline__ void init(const PagedArgs& a) {
    const int lane = threadIdx.x & 63;
    chunk = (a.batch + 63) >> 6;
    m = n = row0 = 0;
    if (a.plan) {
      const int4 sums = ((const int4*)a.plan)[lane];
      lane_units = sums.x;
      lane_cut_units = sums.y;
      lane_cut_tiles = sums.z;
      share = uniform32(sums.w);
    } else {
      int64_t tiles, keys;
      int longest;
      lane_tiles(a, lane, 0, 1, tiles, keys, longest);
      lane_counts(a, lane, 0, 1, tiles, lane64(wave_scan64(tiles), 63), lane64(wave_scan64(keys), 63), longest);
    }
    units = wave_scan(lane_units);
    cut_units = wave_scan(lane_cut_units);
    cut_tiles = wave_scan(lane_cut_tiles);
    total = __builtin_amdgcn_readlane(units, 63);
    total_cut = __builtin_amdgcn_readlane(cut_tiles, 63);
  }

  // Every `step`-th sequence of lane l's from i0 on (large batches: see Line): its tiles of one head, their keys, and the most keys of one;
  // and with the share its units.
  __device__ __forceinline__ void lane_tiles(const PagedArgs& a, int l, int i0, int step, int64_t& tiles, int64_t& keys, int& longest) {
    const int64_t b0 = (int64_t)l * chunk;
    tiles = keys = 0;
    longest = 0;
#pragma unroll 4
    for (int i = i0; i < chunk; i += step) {
      const bool in = b0 + i < a.batch;
      read(a, in ? (int)b0 + i : a.batch - 1, m, n, row0);
      const int t = in ? (int)(((int64_t)m * a.group + QT - 1) / QT) : 0;
      tiles += t;
      keys += t * (int64_t)n;
      longest = t > 0 && n > longest ? n : longest;
    }
  }
  __device__ __forceinline__ void lane_counts(const PagedArgs& a, int l, int i0, int step, int64_t tiles, int64_t all_tiles,
                                              int64_t all_keys, int longest) {
    const int64_t b0 = (int64_t)l * chunk;
    lane_units = lane_cut_units = lane_cut_tiles = 0;
    share = 0x7fffffc0;
    // (more tiles than the rows can make: the offsets do not ascend, and nothing is computed)
    if (all_tiles > (a.grid - 2 * a.workers) / a.kv_heads) return;
    share = find_share(a, (int)tiles, (int)all_tiles * a.kv_heads, all_keys * a.kv_heads, longest);
#pragma unroll 4
    for (int i = i0; i < chunk; i += step) {
      const bool in = b0 + i < a.batch;
      if (chunk > 1) read(a, in ? (int)b0 + i : a.batch - 1, m, n, row0);
      const Counts c = counts(a, in ? m : 0, n);
      lane_units += c.units;
      lane_cut_units += c.cut_units;
      lane_cut_tiles += c.cut_tiles;
    }
  }

  // The smallest share that makes at most `room` units (more than there are tiles).
  __device__ __forceinline__ int64_t least_share(const PagedArgs& a, int tiles, int all_tiles, int64_t all, int room) const {
    int64_t hi = quotient(all, room - all_tiles) + 64, lo = quotient(all, room);  // (units <= keys / share + tiles)
    hi = hi < 0x7fffffff ? hi : 0x7fffffff;
    if (chunk == 1)
      while (hi - lo > 64) {
        const uint32_t mid = (uint32_t)((lo + hi) / 2);
        const int u = __builtin_amdgcn_readlane(wave_scan(tiles * (int)(((uint32_t)n + mid - 1) / mid)), 63) * a.kv_heads;
        if (u <= room) hi = mid; else lo = mid;
      }
    return hi;
  }
  // Tiles that leave a quarter of the workers idle are cut until every worker has a unit.  Where they fill nearly one round of workers or
  // two, what the call takes is estimated in keys per worker: uncut, the rounds that its tiles make (or the longest of them);
  // cut into units of one round or two, their share (of two rounds of unequal units the second ends unevenly: an eighth more) and what writing
  // and joining the parts takes.  Beyond, only tiles that hold more than an even part of all keys are cut.
  __device__ __forceinline__ int find_share(const PagedArgs& a, int tiles, int all_tiles, int64_t all, int longest) const {
    constexpr int JOIN_KEYS = 320;  // (10 us: a worker streams 64 keys in 2 us)
    const int w = a.workers;
    int64_t s;
    if (4 * (int64_t)all_tiles <= 3 * (int64_t)w) {
      s = least_share(a, tiles, all_tiles, all, w);
    } else if (4 * (int64_t)all_tiles <= 7 * (int64_t)w) {
      const int r = 8 * (int64_t)all_tiles <= 7 * (int64_t)w ? 1 : 2;
      s = least_share(a, tiles, all_tiles, all, r * w);
      longest = wave_max(longest);
      const int64_t rounds = quotient(all, all_tiles) * ((all_tiles + w - 1) / w);
      if ((r == 1 ? s : 2 * s + s / 4) + JOIN_KEYS >= (rounds > longest ? rounds : longest)) s = longest;
    } else {
      s = quotient(all, w) + 1;
    }
    s = s > a.min_share ? s : a.min_share;
    return uniform32((int)(s < 0x7fffffc0 ? s : 0x7fffffc0));
  }

  // (u < total)
  __device__ __forceinline__ ManyUnit find(const PagedArgs& a, int u) const {
    const int lane = threadIdx.x & 63;
    const int l = __popcll(__ballot(units <= u));
    int before = __builtin_amdgcn_readlane(units - lane_units, l);
    int slots = __builtin_amdgcn_readlane(cut_units - lane_cut_units, l);
    int cuts = __builtin_amdgcn_readlane(cut_tiles - lane_cut_tiles, l);
    ManyUnit r;
    int b = l * chunk;
    r.b = b;
    if (chunk == 1) {
      r.m = __builtin_amdgcn_readlane(m, l);
      r.n = __builtin_amdgcn_readlane(n, l);
      r.row0 = __builtin_amdgcn_readlane(row0, l);
    } else {
      for (int left = chunk; left > 0; left -= 64) {  // sequences b .. b + 63 of the lane's, one per lane
        Counts c = {};
        int m_ = 0, n_ = 0, r_ = 0;
        if (lane < left && b + lane < a.batch) {
          read(a, b + lane, m_, n_, r_);
          c = counts(a, m_, n_);
        }
        const int iu = wave_scan(c.units), is = wave_scan(c.cut_units), ic = wave_scan(c.cut_tiles);
        const int j = __popcll(__ballot(before + iu <= u));
        if (j < 64) {
          before += __builtin_amdgcn_readlane(iu - c.units, j);
          slots += __builtin_amdgcn_readlane(is - c.cut_units, j);
          cuts += __builtin_amdgcn_readlane(ic - c.cut_tiles, j);
          r.b = b + j;
          r.m = __builtin_amdgcn_readlane(m_, j);
          r.n = __builtin_amdgcn_readlane(n_, j);
          r.row0 = __builtin_amdgcn_readlane(r_, j);
          break;
        }
        before += __builtin_amdgcn_readlane(iu, 63);
        slots += __builtin_amdgcn_readlane(is, 63);
        cuts += __builtin_amdgcn_readlane(ic, 63);
        b += 64;
      }
    }
    r.b = uniform32(r.b);
    r.tiles = uniform32((int)(((int64_t)r.m * a.group + QT - 1) / QT));
    const int pieces = uniform32(counts(a, r.m, r.n).pieces);
    const uint32_t rel = u - before, per_head = (uint32_t)r.tiles * pieces;
    r.h = uniform32(rel / per_head);
    const uint32_t x = rel - r.h * per_head;
    r.piece = uniform32(x / r.tiles);
    r.t = uniform32(x - r.piece * r.tiles);
    const int64_t p0 = (int64_t)r.t * QT, all = (int64_t)r.m * a.group;
    r.pairs = uniform32(all - p0 < QT ? (int)(all - p0) : QT);
    r.lim0 = r.vis = r.n;
    if (a.causal) {
      const int64_t past = (int64_t)r.n - r.m + 1;
      r.lim0 = uniform32(clampi(past + (int)((uint32_t)p0 / a.group), 0, r.n));
      r.vis = uniform32(clampi(past + (int)((uint32_t)(p0 + r.pairs - 1) / a.group), 0, r.n));
    }
    const int size = uniform32((int)((((int64_t)r.n + pieces - 1) / pieces + 63) & ~63ll));  // keys of a piece
    const int64_t k0 = (int64_t)r.piece * size;
    r.k0 = uniform32(k0 < r.vis ? (int)k0 : r.vis);
    r.k1 = uniform32(k0 + size < r.vis ? (int)(k0 + size) : r.vis);
    const int parts = r.vis > size ? (int)(((int64_t)r.vis + size - 1) / size) : 1;
    r.parts = uniform32(pieces > 1 ? parts : 1);
    r.slot = slots + (int)rel;
    r.cut = pieces > 1 ? cuts + r.h * r.tiles + r.t : -1;
    return r;
  }
};

// The record of a tile whose part sg a worker has done, starting at place `at` of the line: parts == 0 unless it began there and goes on.
__device__ __forceinline__ CutTile cut_tile(const PagedArgs& a, const Place& p, const Segment& sg, int64_t at, int64_t share,
                                            int64_t w, int qt) {
  CutTile c = {};
  if (sg.first && !sg.last) {
    c.parts = (int)(quotient(at + sg.cost - 1, share) - w) + 1;
    c.pairs = sg.pairs;
    c.pair0 = p.t * qt;
    c.head = p.h;
    c.row0 = p.s.row0;
    c.slot0 = (int)(2 * w + 1);
    c.next = (int)(2 * w + 2);
    c.step = 2;
  }
  return c;
}

// Rows of the `most` from `key` on that lie before `end`, none without a page.  (In a scalar register: the clamp is a vector
// instruction, and a descriptor made of its result would be a loop over the lanes.)
__device__ __forceinline__ int rows_before(int id, int key, int end, int most) {
  const int left = end - key;
  return uniform32(id < 0 || left < 0 ? 0 : (left < most ? left : most));
}

// Page ids of a sequence, 64 at a time in the lanes of a register: ids outside the cache become -1 (such a page's rows count as
// zeros: nothing is read through a wrong id), and so do entries behind the last one that is needed.
struct PageIds {
  int first, ids;  // ids: lane i holds entry first + i
  __device__ __forceinline__ void fill(const PagedView& c, int b, int entry, int entries) {
    first = entry;
    const int i = entry + (int)(threadIdx.x & 63);
    int id = -1;
    if (i < entries) id = c.table[(int64_t)b * c.table_stride + i];
    ids = (uint32_t)id < c.num_pages ? id : -1;
  }
  __device__ __forceinline__ int get(int entry) const { return __builtin_amdgcn_readlane(ids, entry - first); }
  __device__ __forceinline__ bool holds(int entry) const { return (uint32_t)(entry - first) < 64u; }
};

// pairs of (q row, head) per tile and one-wave workers
constexpr int FEW_PAIRS = 16;
constexpr int MANY_PAIRS = 128;
// The lanes' sums of Line or Units (PagedArgs::plan).
constexpr int PLAN_BYTES = 64 * 16;
hipError_t launch_paged_plan(const PagedArgs& a, int many, hipStream_t stream);
hipError_t launch_paged_few(const PagedArgs& a, int dtype_f32, int d_qk, int d_v, hipStream_t stream);
hipError_t launch_paged_many(const PagedArgs& a, int d_qk, int d_v, hipStream_t stream);
// Adds up the partial results of cut tiles.  many: of the kernel with tiles of MANY_PAIRS.
hipError_t launch_paged_reduce(const PagedArgs& a, int many, int d_v, hipStream_t stream);

// Rotation and appending.
struct RotaryTensor {
  const char* src;
  char* dst;
  int64_t src_stride, dst_stride;  // bytes from row to row (dst: from page to page where `paged`)
  int32_t heads, d, rotate, paged;
};
struct RotaryArgs {
  RotaryTensor t[4];
  int32_t count;
  const double* freq;    // radians per position, rotary / 2 of them
  int32_t rotary, interleaved;
  float scale, sign;     // sign: +1 forward, -1 backward
  const int32_t* pos;    // positions of the rows, or null: places in their sequences
  const int32_t* off;
  int32_t batch, rows;
  int32_t stream;        // nontemporal stores
  PagedView c;           // appending
  const int32_t* ts;     // timestamps of the rows, or null
};
hipError_t launch_rotary(const RotaryArgs& a, int dtype_f32, hipStream_t stream);
hipError_t launch_append(const RotaryArgs& a, int dtype_f32, hipStream_t stream);

}  // namespace hstu
