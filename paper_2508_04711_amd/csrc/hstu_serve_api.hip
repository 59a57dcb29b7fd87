// C ABI of rotary positions, the paged cache and the attention over it: argument checks, division of the work, launches.
// See include/hstu_attn.h for the contract of every entry point.
#include <cmath>

#include "../../include/hstu_attn.h"
#include "hstu_paged.h"
#include "hstu_timing.h"

namespace {

using namespace hstu;

bool dim_ok(int d) { return d == 32 || d == 64 || d == 128; }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
int64_t size_of(int dtype) { return dtype == HSTU_BF16 ? 2 : 4; }
bool stride_ok(int64_t stride, int64_t least, int64_t size) {
  return stride >= least && stride < (1ll << 40) && stride * size % 16 == 0;
}

int check_rotary(const hstu_rotary_desc* r, int head_dim) {
  if (r->rotary_dim < 16 || r->rotary_dim % 16 != 0 || r->rotary_dim > head_dim || !std::isfinite(r->scale))
    return HSTU_ERR_BAD_SHAPE;
  if (r->reserved != 0) return HSTU_ERR_UNSUPPORTED;
  if (!r->inv_freq) return HSTU_ERR_NULL_PTR;
  return (reinterpret_cast<uintptr_t>(r->inv_freq) & 7u) ? HSTU_ERR_MISALIGNED : HSTU_OK;
}

// Shapes of a tensor whose rows are turned (or copied).
int check_rows(const hstu_rotary_tensor* t, int64_t size) {
  if (t->num_heads < 1 || t->num_heads > (1 << 15)) return HSTU_ERR_BAD_SHAPE;
  if (!dim_ok(t->head_dim)) return HSTU_ERR_UNSUPPORTED;
  const int64_t width = (int64_t)t->num_heads * t->head_dim;
  if (!stride_ok(t->src_stride, width, size) || !stride_ok(t->dst_stride, width, size)) return HSTU_ERR_BAD_SHAPE;
  return t->src == t->dst && t->src_stride != t->dst_stride ? HSTU_ERR_BAD_SHAPE : HSTU_OK;
}
int check_row_pointers(const hstu_rotary_tensor* t) {
  if (!t->src || !t->dst) return HSTU_ERR_NULL_PTR;
  return aligned16(t->src) && aligned16(t->dst) ? HSTU_OK : HSTU_ERR_MISALIGNED;
}

// Threads that a launch may have in one direction of its grid.
constexpr int64_t MAX_THREADS = (1ll << 32) - 1;
// Do `rows` rows of head_dim elements fit a launch of the kernel that turns and appends rows (d / 16 threads a row, fp32 d / 8)?
bool rows_fit(int64_t rows, int head_dim, int64_t size) { return (rows + 255) * (head_dim * size / 32) <= MAX_THREADS; }

RotaryTensor tensor_of(const hstu_rotary_tensor* t, int64_t size) {
  RotaryTensor r = {};
  r.src = (const char*)t->src; r.dst = (char*)t->dst;
  r.src_stride = t->src_stride * size; r.dst_stride = t->dst_stride * size;
  r.heads = t->num_heads; r.d = t->head_dim;
  r.rotate = 1;
  return r;
}

// (pointers apart: the workspace query needs none)
int check_cache(const hstu_paged_cache* c) {
  if (!c) return HSTU_ERR_NULL_PTR;
  if (c->batch < 0 || c->num_kv_heads < 1 || c->num_kv_heads > (1 << 15) || c->pages_per_seq < 0 || c->num_pages < 0 || c->num_pages >= (1ll << 31) ||
      c->table_stride < c->pages_per_seq || c->table_stride >= (1ll << 40))
    return HSTU_ERR_BAD_SHAPE;
  if (!dim_ok(c->d_qk) || !dim_ok(c->d_v) || (c->dtype != HSTU_BF16 && c->dtype != HSTU_F32) || c->reserved != 0)
    return HSTU_ERR_UNSUPPORTED;
  if (c->page_size < 16 || c->page_size > 32768 || (c->page_size & (c->page_size - 1)) != 0) return HSTU_ERR_UNSUPPORTED;
  const int64_t rows = (int64_t)c->num_kv_heads * c->page_size, size = size_of(c->dtype);
  if (!stride_ok(c->k_page_stride, rows * c->d_qk, size) || !stride_ok(c->v_page_stride, rows * c->d_v, size))
    return HSTU_ERR_BAD_SHAPE;
  return HSTU_OK;
}
int check_cache_pointers(const hstu_paged_cache* c) {
  if ((c->pages_per_seq > 0 && !c->page_table) || !c->seq_lens) return HSTU_ERR_NULL_PTR;
  if (c->num_pages > 0 && (!c->k_pages || !c->v_pages)) return HSTU_ERR_NULL_PTR;
  return aligned16(c->k_pages) && aligned16(c->v_pages) && aligned16(c->ts_pages) ? HSTU_OK : HSTU_ERR_MISALIGNED;
}

PagedView view_of(const hstu_paged_cache* c) {
  PagedView v = {};
  v.k = (const char*)c->k_pages; v.v = (const char*)c->v_pages;
  v.k_page = c->k_page_stride * size_of(c->dtype);
  v.v_page = c->v_page_stride * size_of(c->dtype);
  v.table = c->page_table; v.table_stride = c->table_stride;
  v.lens = c->seq_lens;
  v.ts = c->ts_pages;
  v.num_pages = (uint32_t)c->num_pages;
  v.ps_log2 = 31 - __builtin_clz((unsigned)c->page_size);
  const int64_t cap = (int64_t)c->pages_per_seq * c->page_size;
  v.cap = cap < MAX_KEYS ? (int32_t)cap : MAX_KEYS;
  return v;
}

// How the attention's work is divided (see hstu_paged.h).
struct Division {
  bool many;
  int whole, workers, grid, min_share, stream;
  bool plan;                   // sums over the sequences come from a kernel of their own
  size_t sums, front, bytes;   // bytes of these; and records of cut tiles; and partial results
};
constexpr int MANY_MEAN = 8;        // pairs per sequence and key/value head beyond which tiles of 128 pairs are the better ones
// Workgroups that run at once: two per CU by registers and LDS, three of the smaller heads (4 x 512..1024 new rows over 4096..16384,
// H = 8, d = 64: 106 us with two, 100 with three, 104 with four; d = 32: 85, 80, 78; 32 x 16..64 rows over 512..4096, d = 64: 48, 43, 52).
int many_workers(const hstu_paged_cache* c) { return c->d_qk + c->d_v <= 160 ? 768 : 512; }
constexpr int MANY_SHARE = 128;
constexpr int FEW_WORKERS = 1024;   // a one-wave worker per SIMD: 768..1536 are within 3 %, 2048 and 512 3 to 5 % behind
constexpr int MIN_SHARE = 64;       // keys that are worth a worker
constexpr int WHOLE_KEYS = 512;     // up to that many keys a tile is one worker's, uncut
constexpr int TEAM_BYTES = 1 << 19; // up to that many bytes of keys and values a tile, and that many tiles, the worker is a
constexpr int TEAM_TILES = 512;     // team of waves, which joins its results itself

// Sequences up to which every worker sums the batch up by itself; beyond, a launch does that once.  In turn without and with it, H = 4,
// d = 64: one new row over 1..256 of 256, 512, 1024, 4096 sequences 12.1 / 14.8, 20.1 / 22.0, 40.1 / 35.9, 253 / 100 us; 32..64 rows over
// up to 1024 of 128 and 256 34.7 / 38.0, 60.0 / 54.0; 16..32 over up to 512 of 512 and 1024 75 / 51, 198 / 87; d = 32, 4096: 2434 / 198.
constexpr int PLAN_FEW = 512, PLAN_MANY = 128;

// Bytes of keys and values from which on the loads are nontemporal: half of the 256 MB of the memory-side cache, which then has nothing
// to keep for the next call.  One new row over 307 MB (64 histories) 61.5 -> 54.4 us, 393 MB 75.8 -> 66.5, 144 MB with the bias 39.5 -> 35.4,
// fp32 36.1 -> 32.5; 95 MB 23.6 either way; teams, which come nowhere near the memory's rate, lose (69 MB 18.2 -> 22.4).  Only where one
// tile of pairs reads a row: 12 new rows over 150 MB 41.0 -> 37.7; several tiles lose (bursts 145 -> 152).
constexpr int64_t STREAM_BYTES = 128 << 20;
constexpr int STREAM_MEAN = 100;    // pairs per sequence and key/value head up to which most sequences have one tile of 128

// false: sizes out of range
bool divide(const hstu_paged_attn_params* p, const hstu_paged_cache* c, Division* d) {
  const int group = p->num_heads / c->num_kv_heads;
  const int64_t cap = view_of(c).cap, pairs = p->new_rows * group;
  const int64_t keys = p->max_kv > 0 && p->max_kv < cap ? p->max_kv : cap;
  // tiles of one head, at most: every sequence with rows may leave one of its tiles with a single pair
  auto tiles_of = [&](int64_t qt) { return (pairs + (qt - 1) * (c->batch < p->new_rows ? c->batch : p->new_rows)) / qt; };
  const bool team = keys * (c->d_qk + c->d_v) * size_of(c->dtype) <= TEAM_BYTES &&
                    tiles_of(FEW_PAIRS) * c->num_kv_heads <= TEAM_TILES;
  // (workgroups of 256 threads; beyond what a launch may have, one-wave workers on cut lines)
  d->many = c->dtype == HSTU_BF16 && !team && pairs > (int64_t)MANY_MEAN * c->batch &&
            (tiles_of(MANY_PAIRS) * c->num_kv_heads + 2 * many_workers(c) + 8) * 256 <= MAX_THREADS;
  const int64_t qt = d->many ? MANY_PAIRS : FEW_PAIRS, tiles = tiles_of(qt);
  // the line of all work, in its own units, has to fit 62 bits, also where every sequence says that all rows are its own
  const double most = (double)c->batch * ((double)pairs / (double)qt + 1.0);
  if ((double)c->num_kv_heads * most * ((double)(cap + 2 * TILE_KEYS) * group + (double)pairs + 256.0) > 4e18) return false;
  const int64_t all = tiles * c->num_kv_heads;
  const int64_t rows = (int64_t)c->batch * keys < c->num_pages * c->page_size ? (int64_t)c->batch * keys : c->num_pages * c->page_size;
  d->stream = rows * c->num_kv_heads * (c->d_qk + c->d_v) * size_of(c->dtype) > STREAM_BYTES &&
              pairs <= (int64_t)STREAM_MEAN * c->batch;
  d->whole = d->many ? keys <= MANY_SHARE : (team ? 2 : (keys <= WHOLE_KEYS && (all + 8) * 64 <= MAX_THREADS ? 1 : 0));
  d->min_share = d->many ? MANY_SHARE : MIN_SHARE;
  d->plan = c->batch > (d->many ? PLAN_MANY : PLAN_FEW);
  d->sums = d->plan ? PLAN_BYTES : 0;
  if (d->many) {
    // every uncut tile is a unit, and cut ones make at most twice as many as there are workers, two or more a tile (see Units)
    d->workers = many_workers(c);
    d->grid = (int)((all + 2 * d->workers + 7) / 8 * 8);
    d->front = d->sums + (d->whole ? 0 : align_up((size_t)d->workers * sizeof(CutTile), 256));
    d->bytes = d->whole ? d->front : d->front + (size_t)(2 * d->workers) * qt * c->d_v * sizeof(float);
    return true;
  }
  int64_t workers = all;
  if (!d->whole) {
    const double most = (double)all * (double)(keys + 2 * TILE_KEYS) / MIN_SHARE + 1.0;
    workers = most < FEW_WORKERS ? (int64_t)most : FEW_WORKERS;
  }
  d->workers = d->grid = (int)((workers + 7) / 8 * 8);
  d->front = d->sums + (d->whole ? 0 : align_up((size_t)d->workers * sizeof(CutTile), 256));
  d->bytes = d->whole ? d->front : d->front + (size_t)d->workers * 2 * (size_t)qt * c->d_v * sizeof(float);
  return true;
}

int check_paged(const hstu_paged_attn_params* p, const hstu_paged_cache* c, Division* d) {
  if (!p) return HSTU_ERR_NULL_PTR;
  const int rc = check_cache(c);
  if (rc != HSTU_OK) return rc;
  if (p->num_heads < 1 || p->num_heads > (1 << 15) || p->num_heads % c->num_kv_heads != 0 || p->max_len < 1 || !std::isfinite(p->alpha) || p->max_kv < 0 ||
      p->new_rows < 0 || p->new_rows >= (1ll << 31) || p->new_rows * (p->num_heads / c->num_kv_heads) >= (1ll << 31) - 256)
    return HSTU_ERR_BAD_SHAPE;
  if (p->out_dtype != c->dtype && p->out_dtype != HSTU_F32) return HSTU_ERR_UNSUPPORTED;
  return divide(p, c, d) ? HSTU_OK : HSTU_ERR_BAD_SHAPE;
}

}  // namespace

extern "C" {

int hstu_rotary(const hstu_rotary_desc* rotary, int32_t backward, int32_t dtype, int32_t batch, int64_t rows,
                int32_t num_tensors, const hstu_rotary_tensor* tensors, const int32_t* positions,
                const int32_t* seq_offsets, void* hip_stream) {
  if (!rotary || !tensors) return HSTU_ERR_NULL_PTR;
  if (batch < 0 || rows < 0 || rows >= (1ll << 31) || num_tensors < 1 || num_tensors > 4) return HSTU_ERR_BAD_SHAPE;
  if (dtype != HSTU_BF16 && dtype != HSTU_F32) return HSTU_ERR_UNSUPPORTED;
  RotaryArgs a = {};
  for (int i = 0; i < num_tensors; ++i) {
    int rc = check_rows(&tensors[i], size_of(dtype));
    if (rc == HSTU_OK) rc = check_rotary(rotary, tensors[i].head_dim);
    if (rc != HSTU_OK) return rc;
    if (!rows_fit(rows, tensors[i].head_dim, size_of(dtype))) return HSTU_ERR_BAD_SHAPE;
    a.t[i] = tensor_of(&tensors[i], size_of(dtype));
  }
  if (rows == 0 || (!positions && batch == 0)) return HSTU_OK;
  if (!positions && !seq_offsets) return HSTU_ERR_NULL_PTR;
  for (int i = 0; i < num_tensors; ++i)
    if (const int rc = check_row_pointers(&tensors[i])) return rc;
  for (int i = 0; i < num_tensors; ++i)  // a tensor may be turned in place, not into another one's place
    for (int j = 0; j < num_tensors; ++j)
      if (i != j && (tensors[i].dst == tensors[j].dst || tensors[i].dst == tensors[j].src)) return HSTU_ERR_BAD_SHAPE;
  a.count = num_tensors;
  a.freq = rotary->inv_freq;
  a.rotary = rotary->rotary_dim; a.interleaved = rotary->interleaved ? 1 : 0;
  a.scale = rotary->scale; a.sign = backward ? -1.f : 1.f;
  a.pos = positions; a.off = seq_offsets;
  a.batch = batch; a.rows = (int32_t)rows;
  int64_t written = 0;
  for (int i = 0; i < num_tensors; ++i) written += rows * tensors[i].num_heads * tensors[i].head_dim * size_of(dtype);
  a.stream = written > (256ll << 20);
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  TimedLaunch timed(14, stream);
  return launch_rotary(a, dtype == HSTU_F32, stream) == hipSuccess ? HSTU_OK : HSTU_ERR_HIP;
}

int hstu_cache_append(const hstu_paged_cache* cache, const hstu_rotary_desc* rotary, int64_t new_rows,
                      const hstu_rotary_tensor* q, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                      const int32_t* timestamps, const int32_t* seq_offsets, void* hip_stream) {
  int rc = check_cache(cache);
  if (rc != HSTU_OK) return rc;
  const int64_t size = size_of(cache->dtype);
  if (new_rows < 0 || new_rows >= (1ll << 31) || !rows_fit(new_rows, cache->d_qk > cache->d_v ? cache->d_qk : cache->d_v, size))
    return HSTU_ERR_BAD_SHAPE;
  if (rotary && (rc = check_rotary(rotary, cache->d_qk)) != HSTU_OK) return rc;
  if (!stride_ok(k_stride, (int64_t)cache->num_kv_heads * cache->d_qk, size) ||
      !stride_ok(v_stride, (int64_t)cache->num_kv_heads * cache->d_v, size))
    return HSTU_ERR_BAD_SHAPE;
  if (q && ((rc = check_rows(q, size)) != HSTU_OK)) return rc;
  if (q && q->head_dim != cache->d_qk) return HSTU_ERR_BAD_SHAPE;
  if (cache->batch == 0 || new_rows == 0) return HSTU_OK;
  if (!k || !v || !seq_offsets) return HSTU_ERR_NULL_PTR;
  // (a cache without pages has no address for timestamps either, and no place for any)
  if (cache->num_pages > 0 && (cache->ts_pages != nullptr) != (timestamps != nullptr)) return HSTU_ERR_NULL_PTR;
  if (!aligned16(k) || !aligned16(v)) return HSTU_ERR_MISALIGNED;
  if ((rc = check_cache_pointers(cache)) != HSTU_OK) return rc;
  if (q && (rc = check_row_pointers(q)) != HSTU_OK) return rc;
  if (q && (q->dst == k || q->dst == v)) return HSTU_ERR_BAD_SHAPE;  // (may be q itself, not what others still read)
  RotaryArgs a = {};
  RotaryTensor& tk = a.t[a.count++];
  tk.src = (const char*)k; tk.src_stride = k_stride * size;
  tk.dst = (char*)cache->k_pages; tk.dst_stride = cache->k_page_stride * size;
  tk.heads = cache->num_kv_heads; tk.d = cache->d_qk;
  tk.rotate = rotary != nullptr; tk.paged = 2;  // (the one that takes the timestamps along)
  RotaryTensor& tv = a.t[a.count++];
  tv.src = (const char*)v; tv.src_stride = v_stride * size;
  tv.dst = (char*)cache->v_pages; tv.dst_stride = cache->v_page_stride * size;
  tv.heads = cache->num_kv_heads; tv.d = cache->d_v;
  tv.paged = 1;
  if (q) {
    a.t[a.count] = tensor_of(q, size);
    a.t[a.count++].rotate = rotary != nullptr;
  }
  if (rotary) {
    a.freq = rotary->inv_freq;
    a.rotary = rotary->rotary_dim; a.interleaved = rotary->interleaved ? 1 : 0;
    a.scale = rotary->scale;
  }
  a.sign = 1.f;
  a.off = seq_offsets;
  a.batch = cache->batch; a.rows = (int32_t)new_rows;
  a.c = view_of(cache);
  a.ts = timestamps;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  TimedLaunch timed(15, stream);
  return launch_append(a, cache->dtype == HSTU_F32, stream) == hipSuccess ? HSTU_OK : HSTU_ERR_HIP;
}

size_t hstu_paged_attn_workspace_bytes(const hstu_paged_attn_params* params, const hstu_paged_cache* cache) {
  Division d;
  if (check_paged(params, cache, &d) != HSTU_OK) return 0;
  return d.bytes > 256 ? d.bytes : 256;
}

int hstu_paged_attn_fwd(const hstu_paged_attn_params* params, const hstu_paged_cache* cache, const hstu_ts_bias* bias,
                        const void* q, int64_t q_stride, const int32_t* seq_offsets, void* o, void* workspace,
                        size_t workspace_bytes, void* hip_stream) {
  Division d;
  int rc = check_paged(params, cache, &d);
  if (rc != HSTU_OK) return rc;
  const int64_t size = size_of(cache->dtype);
  if (!stride_ok(q_stride, (int64_t)params->num_heads * cache->d_qk, size)) return HSTU_ERR_BAD_SHAPE;
  if (bias && (bias->num_buckets < 1 || bias->num_buckets > MAX_TS_BUCKETS || bias->groups_log2 < 0 || bias->groups_log2 > 8))
    return HSTU_ERR_BAD_SHAPE;
  if (cache->batch == 0 || params->new_rows == 0) return HSTU_OK;
  if (!q || !o || !seq_offsets || !workspace) return HSTU_ERR_NULL_PTR;
  if (bias && (!bias->timestamps || !bias->ts_weights || (cache->num_pages > 0 && !cache->ts_pages))) return HSTU_ERR_NULL_PTR;
  if ((rc = check_cache_pointers(cache)) != HSTU_OK) return rc;
  if (!aligned16(q) || !aligned16(o) || !aligned16(workspace)) return HSTU_ERR_MISALIGNED;
  if (workspace_bytes < d.bytes) return HSTU_ERR_WORKSPACE_TOO_SMALL;
  PagedArgs a = {};
  a.c = view_of(cache);
  a.q = (const char*)q; a.q_stride = q_stride * size;
  a.off = seq_offsets;
  if (bias) {
    a.ts_q = bias->timestamps; a.ts_w = bias->ts_weights;
    a.nb = bias->num_buckets; a.f = bias->groups_log2;
  }
  a.o = o;
  a.plan = d.plan ? workspace : nullptr;
  a.cut = (CutTile*)((char*)workspace + d.sums);
  a.partial = (float*)((char*)workspace + d.front);
  a.batch = cache->batch; a.rows = (int32_t)params->new_rows;
  a.heads = params->num_heads; a.kv_heads = cache->num_kv_heads; a.group = params->num_heads / cache->num_kv_heads;
  a.causal = params->causal ? 1 : 0;
  a.out_f32 = params->out_dtype == HSTU_F32;
  a.alpha = params->alpha; a.inv_n = 1.f / (float)params->max_len;
  a.workers = d.workers; a.grid = d.grid; a.whole = d.whole; a.min_share = d.min_share;
  a.stream = d.stream;
  a.records = d.many && !d.whole ? d.workers : 0;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (d.plan) {
    TimedLaunch timed(3, stream);
    if (launch_paged_plan(a, d.many, stream) != hipSuccess) return HSTU_ERR_HIP;
  }
  {
    TimedLaunch timed(16, stream);
    const hipError_t e = d.many ? launch_paged_many(a, cache->d_qk, cache->d_v, stream)
                                : launch_paged_few(a, cache->dtype == HSTU_F32, cache->d_qk, cache->d_v, stream);
    if (e != hipSuccess) return HSTU_ERR_HIP;
  }
  if (d.whole) return HSTU_OK;
  TimedLaunch timed(17, stream);
  return launch_paged_reduce(a, d.many, cache->d_v, stream) == hipSuccess ? HSTU_OK : HSTU_ERR_HIP;
}

}  // extern "C"
