// What the kernels of the paged cache share (not part of the C ABI): the view of a cache, and the schedule of the attention of
// new rows over it.
#pragma once
#include "hstu_common.h"

namespace hstu {

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
  CutTile* cut;               // one per worker
  float* partial;             // two slots per worker
  int32_t batch, rows, heads, kv_heads, group;
  int32_t causal, out_f32;
  float alpha, inv_n;
  int32_t workers;            // a multiple of 8
  int32_t whole;              // 1: every worker takes one tile, uncut; 2: ... and is a team of waves
  int32_t min_share;          // keys a worker takes at least
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
// HELD: where every lane has one sequence only, it is kept (three registers) and not read again.
template <int QT, bool HELD>
struct Line {
  int chunk;
  int64_t incl, sum;  // of the lane's sequences and all before them; of the lane's alone
  int64_t total;
  int m, n, row0;     // chunk 1: the lane's sequence

  __device__ __forceinline__ void init(const PagedArgs& a) {
    const int lane = threadIdx.x & 63;
    chunk = (a.batch + 63) >> 6;
    sum = 0;
    m = n = row0 = 0;
    const int64_t b0 = (int64_t)lane * chunk;
    for (int i = 0; i < chunk; ++i)
      if (b0 + i < a.batch) {
        const SeqWork s = read_work<QT>(a, (int)b0 + i);
        sum += s.cost;
        m = s.m; n = s.n; row0 = s.row0;
      }
    sum *= a.kv_heads;
    incl = wave_scan64(sum);
    total = lane64(incl, 63);
  }

  // The work of sequence b (uniform): from the lane that has read it already where every lane has one.
  __device__ __forceinline__ SeqWork work(const PagedArgs& a, int b) const {
    if (!HELD || chunk > 1) return read_work<QT>(a, b);
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

// What the reduce kernel has to know of the tile that a worker began and did not finish.  Every worker writes one.
struct CutTile {
  int32_t parts;   // workers the tile reaches into, or 0: no such tile
  int32_t pairs, pair0, head, row0, pad[3];
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
  }
  return c;
}

// Rows of the 16 from `key` on that lie before `end`, none without a page.  (In a scalar register: the clamp is a vector
// instruction, and a descriptor made of its result would be a loop over the lanes.)
__device__ __forceinline__ int rows_before(int id, int key, int end) {
  const int left = end - key;
  return uniform32(id < 0 || left < 0 ? 0 : (left < 16 ? left : 16));
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
  PagedView c;           // appending
  const int32_t* ts;     // timestamps of the rows, or null
};
hipError_t launch_rotary(const RotaryArgs& a, int dtype_f32, hipStream_t stream);
hipError_t launch_append(const RotaryArgs& a, int dtype_f32, hipStream_t stream);

}  // namespace hstu
