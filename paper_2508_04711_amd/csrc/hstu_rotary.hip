// Rotary positions on jagged rows (forward and backward), and appending rows to a paged cache with the rotation on the way.
//
// The pairs (a, b) of a head's first `rotary` elements, (j, j + rotary/2) or interleaved (2j, 2j + 1), are turned by the angle
// position * freq[j]:  y_a = x_a c - x_b s,  y_b = x_b c + x_a s,  c, s = scale * (cos, sin).  The map is linear and, up to
// the scale, orthogonal: its gradient is the same turn by the opposite angle.
//
// Bound by reading and writing the rows once.  A thread takes eight pairs' worth of a row (two 16-byte chunks half the turned part
// apart, which hold whole pairs in either layout; fp32: four pairs) and works their angles out once for up to four heads of a tensor, whose eight loads are in flight
// together.  Angles: position * frequency / 2 pi in double precision, less the nearest whole turn, is exact to 1e-10 of a turn at
// a million radians (1e-7 at the largest int32 position), where 32 bits lose a tenth of a turn (whole turns); the sine and cosine of what remains, at most an eighth of a turn after
// taking off quarter turns, are their Taylor polynomials in fp32 (error below 2^-27).
//
// The rows are read with nontemporal loads (they are not needed again: q and k of 37117 rows, H = 4, and their gradients 64.7 -> 62.5 us),
// and where a call writes more than the 256 MB of the memory-side cache, written so too (96016 rows, H = 8: 292 -> 278 us; appends, whose pages the
// attention reads next, lose: 48.8 -> 63.6).
#include "hstu_mfma.h"
#include "hstu_paged.h"

namespace hstu {

namespace {

constexpr int ROT_THREADS = 256;
constexpr int ROT_HEADS = 4;  // heads a thread does

// The sequence that row belongs to (the last one with off[b] <= row), found by the whole wave together: 64 probes a step.
// row: the same in every lane.
__device__ __forceinline__ int find_sequence(const int32_t* off, int batch, int row) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = batch;
  while (n > 1) {
    const int step = (n + 63) >> 6;
    const int64_t i = (int64_t)lane * step;
    const bool le = i < n && off[lo + i] <= row;
    const int c = __popcll(__ballot(le));
    const int j = c > 0 ? c - 1 : 0;
    lo += j * step;
    n = n - j * step < step ? n - j * step : step;
    lo = __builtin_amdgcn_readfirstlane(lo);
    n = __builtin_amdgcn_readfirstlane(n);
  }
  return lo;
}

// The same for the rows row0 + (lane >> shift): one search for the first, whose followers are looked for among the next 64.
__device__ __forceinline__ int find_sequences(const int32_t* off, int batch, int row0, int rows, int shift) {
  const int lane = threadIdx.x & 63;
  const int b0 = find_sequence(off, batch, row0);
  const int64_t i = (int64_t)b0 + 1 + lane;
  const int next = i < batch ? off[i] : 0x7fffffff;  // first rows of the sequences behind b0
  int b = b0;
  for (int r = 0; r < 64 >> shift; ++r) {
    if (r >= rows - row0) break;
    const int row = row0 + r;
    const int past = __popcll(__ballot(next <= row));
    const int x = past < 64 ? b0 + past : find_sequence(off, batch, row);
    if (lane >> shift == r) b = x;
  }
  return b;
}

// cos and sin of `angle` radians.
__device__ __forceinline__ void turn_of(double angle, float scale, float sign, float& c, float& s) {
  double t = angle * 0.15915494309189533577;  // 1 / (2 pi)
  t = (t - __builtin_rint(t)) * 4.0;  // quarter turns, -2 .. 2
  const double near = __builtin_rint(t);
  const int q = (int)near & 3;
  const float y = (float)(t - near) * 1.5707963267948966f;
  const float z = y * y;
  float sn = 2.7557319e-6f;             // 1/9!
  sn = __builtin_fmaf(sn, z, -1.9841270e-4f);
  sn = __builtin_fmaf(sn, z, 8.3333333e-3f);
  sn = __builtin_fmaf(sn, z, -1.6666667e-1f);
  sn = __builtin_fmaf(sn * z, y, y);
  float cs = -2.7557319e-7f;            // -1/10!
  cs = __builtin_fmaf(cs, z, 2.4801587e-5f);
  cs = __builtin_fmaf(cs, z, -1.3888889e-3f);
  cs = __builtin_fmaf(cs, z, 4.1666667e-2f);
  cs = __builtin_fmaf(cs, z, -0.5f);
  cs = __builtin_fmaf(cs, z, 1.f);
  const float a = (q & 1) ? sn : cs, b = (q & 1) ? cs : sn;  // q = 1: (cos, sin) = (-sn, cs); 2: (-cs, -sn); 3: (sn, -cs)
  c = scale * ((q == 1 || q == 2) ? -a : a);
  s = scale * sign * (q >= 2 ? -b : b);
}

template <bool F32>
struct Chunk {  // 16 bytes of a row
  static constexpr int N = F32 ? 4 : 8;
  u32x4 w;
  __device__ __forceinline__ float get(int e) const {
    const uint32_t x = w[F32 ? e : e >> 1];  // (a value: a bit cast of the vector's element itself yields its first one)
    return __builtin_bit_cast(float, F32 ? x : ((e & 1) ? x & 0xffff0000u : x << 16));
  }
  __device__ __forceinline__ void set(const float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (F32) {
        w[i] = __builtin_bit_cast(uint32_t, x[i]);
      } else {
        bf16x2 t;
        t[0] = (__bf16)x[2 * i];
        t[1] = (__bf16)x[2 * i + 1];
        w[i] = __builtin_bit_cast(uint32_t, t);
      }
    }
  }
};

// Rows of one tensor (blockIdx.y: the tensor and four of its heads).  A row of a head is d / (2 N) threads wide, each of which
// takes the chunks c0 and c1 of it.
template <bool F32, bool INTER, bool APPEND, bool STREAM>
__global__ void __launch_bounds__(ROT_THREADS) rotary_kernel(RotaryArgs a) {
  typedef Chunk<F32> C;
  constexpr int N = C::N;
  int u = blockIdx.y, x = 0;
  while (u >= (a.t[x].heads + ROT_HEADS - 1) / ROT_HEADS) {
    u -= (a.t[x].heads + ROT_HEADS - 1) / ROT_HEADS;
    ++x;
  }
  const RotaryTensor& t = a.t[x];
  const int head0 = u * ROT_HEADS, heads = t.heads - head0 < ROT_HEADS ? t.heads - head0 : ROT_HEADS;
  const int wide = t.d / (2 * N), shift = 31 - __builtin_clz((unsigned)wide);  // (a power of two)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t first = (int64_t)blockIdx.x * (ROT_THREADS >> shift) + wave * (64 >> shift);
  if (first >= a.rows) return;
  const int row0 = (int)first, row = row0 + (lane >> shift), c = lane & (wide - 1);
  const bool in = lane >> shift < a.rows - row0;

  int pos = 0, b = 0;
  bool on = in;
  if (a.pos) {
    if (in) pos = a.pos[row];
  } else {
    b = find_sequences(a.off, a.batch, row0, a.rows, shift);
    // (rows outside every sequence are left alone)
    int s, e;
    seq_range(a.off, b, a.rows, s, e);
    on = in && row >= s && row < e;
    pos = row - s;
    if constexpr (APPEND) {
      // Lengths and offsets count as the attention counts them, wrong ones too: a row's place is the one that the attention takes for its
      // own.  (A sequence without entries has no places; its rows are turned by the positions that its length says.)
      const int64_t n = clampi(a.c.lens[b], 0, a.c.cap > 0 ? a.c.cap : MAX_KEYS);
      pos = (int)(n - e + row);
    }
  }
  // where the row goes
  char* dst = t.dst + (int64_t)row * t.dst_stride + (int64_t)head0 * t.d * (F32 ? 4 : 2);
  int64_t dst_head = (int64_t)t.d * (F32 ? 4 : 2);
  if constexpr (APPEND) {
    if (t.paged) {
      uint32_t id = 0;
      const bool room = on && pos >= 0 && pos < a.c.cap;
      if (room) id = (uint32_t)a.c.table[(int64_t)b * a.c.table_stride + (pos >> a.c.ps_log2)];
      on = room && id < a.c.num_pages;
      const int slot = pos & ((1 << a.c.ps_log2) - 1);
      if (on && t.paged == 2 && head0 == 0 && c == 0 && a.ts) a.c.ts[((int64_t)id << a.c.ps_log2) + slot] = a.ts[row];
      dst_head <<= a.c.ps_log2;
      dst = t.dst + (int64_t)id * t.dst_stride + head0 * dst_head + (int64_t)slot * t.d * (F32 ? 4 : 2);
    }
  }
  if (!on) return;
  const char* src = t.src + (int64_t)row * t.src_stride + (int64_t)head0 * t.d * (F32 ? 4 : 2);
  const int64_t src_head = (int64_t)t.d * (F32 ? 4 : 2);

  // The row's chunks: of the turned part, and of the rest (or of a row that is not turned), a thread takes one of the first half and the
  // one at its place in the second half.
  const int pairs = t.rotate ? a.rotary / (2 * N) : 0;  // threads that turn
  const bool turned = c < pairs;
  if (!turned && t.src == t.dst) return;  // in place: what is not turned stays
  const int c0 = turned ? c : pairs + c, c1 = turned ? c + pairs : wide + c;
  C p[ROT_HEADS], q[ROT_HEADS];
#pragma unroll
  for (int h = 0; h < ROT_HEADS; ++h)
    if (h < heads) {
      p[h].w = __builtin_nontemporal_load((const u32x4*)(src + h * src_head + c0 * 16));
      q[h].w = __builtin_nontemporal_load((const u32x4*)(src + h * src_head + c1 * 16));
    }
  if (turned) {
    float cs[N], sn[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int j = !INTER ? c * N + e : (e < N / 2 ? c0 * (N / 2) + e : c1 * (N / 2) + e - N / 2);  // (interleaved: a chunk's pairs are its own)
      turn_of((double)pos * a.freq[j], a.scale, a.sign, cs[e], sn[e]);
    }
#pragma unroll
    for (int h = 0; h < ROT_HEADS; ++h)
      if (h < heads) {
        float y0[N], y1[N];
        if constexpr (INTER) {
#pragma unroll
          for (int e = 0; e < N / 2; ++e) {
            const float u0 = p[h].get(2 * e), u1 = p[h].get(2 * e + 1), v0 = q[h].get(2 * e), v1 = q[h].get(2 * e + 1);
            y0[2 * e] = u0 * cs[e] - u1 * sn[e];
            y0[2 * e + 1] = u1 * cs[e] + u0 * sn[e];
            y1[2 * e] = v0 * cs[N / 2 + e] - v1 * sn[N / 2 + e];
            y1[2 * e + 1] = v1 * cs[N / 2 + e] + v0 * sn[N / 2 + e];
          }
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const float u0 = p[h].get(e), u1 = q[h].get(e);
            y0[e] = u0 * cs[e] - u1 * sn[e];
            y1[e] = u1 * cs[e] + u0 * sn[e];
          }
        }
        p[h].set(y0);
        q[h].set(y1);
      }
  }
#pragma unroll
  for (int h = 0; h < ROT_HEADS; ++h)
    if (h < heads) {
      u32x4* d0 = (u32x4*)(dst + h * dst_head + c0 * 16);
      u32x4* d1 = (u32x4*)(dst + h * dst_head + c1 * 16);
      if constexpr (STREAM) {
        __builtin_nontemporal_store(p[h].w, d0);
        __builtin_nontemporal_store(q[h].w, d1);
      } else {
        *d0 = p[h].w;
        *d1 = q[h].w;
      }
    }
}

template <bool APPEND>
hipError_t launch_rows(const RotaryArgs& a, int f32, hipStream_t stream) {
  int units = 0, wide = 1;
  for (int x = 0; x < a.count; ++x) {
    units += (a.t[x].heads + ROT_HEADS - 1) / ROT_HEADS;
    const int w = a.t[x].d / (f32 ? 8 : 16);
    wide = w > wide ? w : wide;
  }
  const int64_t per = ROT_THREADS / wide;
  const dim3 grid((unsigned)((a.rows + per - 1) / per), (unsigned)units), block(ROT_THREADS);
#define HSTU_ROWS(F32, INTER)                                                                                       \
  do {                                                                                                             \
    if (!APPEND && a.stream) hipLaunchKernelGGL((rotary_kernel<F32, INTER, APPEND, !APPEND>), grid, block, 0, stream, a); \
    else hipLaunchKernelGGL((rotary_kernel<F32, INTER, APPEND, false>), grid, block, 0, stream, a);                 \
  } while (0)
  if (f32) {
    if (a.interleaved) HSTU_ROWS(true, true); else HSTU_ROWS(true, false);
  } else {
    if (a.interleaved) HSTU_ROWS(false, true); else HSTU_ROWS(false, false);
  }
#undef HSTU_ROWS
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, int dtype_f32, hipStream_t stream) {
  return launch_rows<false>(a, dtype_f32, stream);
}
hipError_t launch_append(const RotaryArgs& a, int dtype_f32, hipStream_t stream) {
  return launch_rows<true>(a, dtype_f32, stream);
}

}  // namespace hstu
