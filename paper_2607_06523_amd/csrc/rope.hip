// Rotary positions, and new tokens into the pages of a dense cache, gfx950.
//
// Pair i of a head at position p turns by the angle p f_i:
//   a' = m (a cos - b sin),  b' = m (b cos + a sin).
// Angles are float64: at position 2^20 a float32 angle is off by 2^-4.  Each
// workgroup works the sines and cosines of its rows out once, into LDS (64 pairs of a row,
// against 64 x 40 rotations that read them): the angle is brought
// into [-pi/4, pi/4] in float64 and the Taylor polynomials there are float64 for
// float32 outputs, float32 for outputs of 16 bits (off by 2^-23 where those have 2^-11).
// Then its threads stream pieces of 16 bytes.  Bound by HBM: what a call of many rows
// writes goes past the caches (16384 rows of 40 heads of 128 turned in 60 us, 5.6 TB/s,
// against 64 with plain stores; a copy of them past the caches takes 59; appended with 8 heads of values 81 against 83, 8100 rows of
// seven prompts 43 against 45).
#include <algorithm>

#include "internal.h"
#include "rows_dev.h"

namespace dwkv {
namespace {

constexpr int kRT = 256;                 // threads of a workgroup
constexpr int kRows = 2;                 // rows of a workgroup, at most
constexpr int kSlots = 16;               // slots of a workgroup that fills pages

enum Pairs { HALF = 0, PART = 1, NEXT = 2 };   // (i, n + i) of all channels, of some; (2i, 2i + 1)

// sin and cos of x.  x - n pi/2 in two steps (n pi/2's upper part is exact in the
// fused product), then Taylor: to x^13 and x^14 in float64 (below 2^-45 on
// [-pi/4, pi/4]), to x^9 and x^8 in float32 (2^-28 and 2^-25).
template <bool FULL>
__device__ __forceinline__ void sin_cos(double x, double& s, double& c) {
  const double n = __builtin_rint(x * 0.63661977236758134308);
  double r = __builtin_fma(n, -1.57079632679489655800, x);
  r = __builtin_fma(n, -6.12323399573676603587e-17, r);
  double p, q;
  if constexpr (FULL) {
    const double z = r * r;
    p = 1.0 / 6227020800.0;
    p = __builtin_fma(p, z, -1.0 / 39916800.0);
    p = __builtin_fma(p, z, 1.0 / 362880.0);
    p = __builtin_fma(p, z, -1.0 / 5040.0);
    p = __builtin_fma(p, z, 1.0 / 120.0);
    p = __builtin_fma(p, z, -1.0 / 6.0);
    p = __builtin_fma(p * z, r, r);
    q = -1.0 / 87178291200.0;
    q = __builtin_fma(q, z, 1.0 / 479001600.0);
    q = __builtin_fma(q, z, -1.0 / 3628800.0);
    q = __builtin_fma(q, z, 1.0 / 40320.0);
    q = __builtin_fma(q, z, -1.0 / 720.0);
    q = __builtin_fma(q, z, 1.0 / 24.0);
    q = __builtin_fma(q, z, -0.5);
    q = __builtin_fma(q, z, 1.0);
  } else {
    const float f = (float)r, z = f * f;
    float u = 1.f / 362880.f;
    u = __builtin_fmaf(u, z, -1.f / 5040.f);
    u = __builtin_fmaf(u, z, 1.f / 120.f);
    u = __builtin_fmaf(u, z, -1.f / 6.f);
    p = __builtin_fmaf(u * z, f, f);
    float v = 1.f / 40320.f;
    v = __builtin_fmaf(v, z, -1.f / 720.f);
    v = __builtin_fmaf(v, z, 1.f / 24.f);
    v = __builtin_fmaf(v, z, -0.5f);
    q = __builtin_fmaf(v, z, 1.f);
  }
  const int k = (int)(long long)n & 3;
  const double u = k & 1 ? q : p, v = k & 1 ? p : q;
  s = k & 2 ? -u : u;
  c = (k + 1) & 2 ? -v : v;
}

// (cos, sin) of row r's pair i at cs[r * entries + i], already scaled.  PART: an entry for each
// of a pair's channels, (cos, -sin) for the first.
template <int P>
__device__ __forceinline__ int entries(int np) {
  return P == PART ? 2 * np : np;
}
template <int P, int TO>
__device__ __forceinline__ void fill_table(float2* cs, const RopeSpec& t, const int* pos, int rows) {
  for (int u = threadIdx.x; u < rows * t.n_pairs; u += kRT) {
    const int r = u / t.n_pairs, i = u - r * t.n_pairs;
    double s, c;
    sin_cos<TO == DWKV_F32>((double)pos[r] * t.freq[i], s, c);
    const float2 of = make_float2((float)(c * t.scale), (float)(s * (t.inverse ? -(double)t.scale : (double)t.scale)));
    if constexpr (P == PART) {
      cs[u + r * t.n_pairs] = make_float2(of.x, -of.y);
      cs[u + (r + 1) * t.n_pairs] = of;
    } else {
      cs[u] = of;
    }
  }
}

__device__ __forceinline__ void turn(float& a, float& b, float2 cs) {
  const float x = a, y = b;
  a = __builtin_fmaf(x, cs.x, -(y * cs.y));
  b = __builtin_fmaf(y, cs.x, x * cs.y);
}

// A head falls into pieces of eight channels; halves of whole heads into pieces of eight pairs.
template <int P>
__device__ __forceinline__ int pieces(int d) {
  return P == HALF ? d / 16 : d / 8;
}

// Piece a of a head, turned, to put(channel, eight numbers), in 16-byte pieces.  Where the
// halves end within the head, a piece has its channels and reads what they pair with once
// more, as the stores of a wave then cover whole lines: 16384 rows of 40 heads of 128,
// the first 48 or 42 channels turned, take 66 and 75 us; in pieces of pairs 105 and 282.
// edge: the first or the last head of all, where eight numbers from within the head may
// reach past the rows' memory.
template <int P, int TI, class Put>
__device__ __forceinline__ void turn_piece(const row_t<TI>* x, int a, int np, bool edge, const float2* cs, Put put) {
  if constexpr (P == NEXT) {
    float8_t v = load8<TI>(x + 8 * a);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (4 * a + i < np) {
        float lo = v[2 * i], hi = v[2 * i + 1];
        turn(lo, hi, cs[4 * a + i]);
        v[2 * i] = lo;
        v[2 * i + 1] = hi;
      }
    put(8 * a, v);
  } else if constexpr (P == HALF) {
    float8_t lo = load8<TI>(x + 8 * a), hi = load8<TI>(x + np + 8 * a);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float u = lo[i], v = hi[i];
      turn(u, v, cs[8 * a + i]);
      lo[i] = u;
      hi[i] = v;
    }
    put(8 * a, lo);
    put(np + 8 * a, hi);
  } else {
    typedef typename AnyPlace<TI>::eight any8;
    const int c = 8 * a;
    const bool low = c < np, cross = low && c + 8 > np, alone = cross && edge;    // cross: in both halves
    // both loads on their way before anything waits for one
    const row8_t<TI> own = *reinterpret_cast<const row8_t<TI>*>(x + c);
    const any8 first = *reinterpret_cast<const any8*>(x + (alone || c >= 2 * np ? c : low ? c + np : c - np));
    any8 back = first;
    if (cross) {
      if (alone) {
#pragma unroll
        for (int i = 0; i < 8; ++i) back[i] = x[c + i < np ? c + i + np : c + i < 2 * np ? c + i - np : 0];
      } else {
        back = *reinterpret_cast<const any8*>(x + c - np);
      }
    }
    float8_t v = __builtin_convertvector(own, float8_t);
    if (c < 2 * np) {
      const float8_t f = __builtin_convertvector(first, float8_t), b = __builtin_convertvector(back, float8_t);
      const float2* t = cs + c;
      const int turns = alone ? 0 : low ? np - c : 8;            // numbers of `first` that count
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < 2 * np) v[i] = __builtin_fmaf(v[i], t[i].x, (i < turns ? f[i] : b[i]) * t[i].y);
    }
    put(c, v);
  }
}

// Pieces of heads that a workgroup has at a time.  PART in place: whole heads, which are all read
// before any is stored.
template <int P>
__device__ __forceinline__ int pieces_at_once(int A, bool in_place) {
  return P == PART && in_place ? kRT / A * A : kRT;
}

// The pieces of `rows` rows, `per` in each: from(row, head) to to(row, head, channel, eight numbers).
template <int P, int TI, class From, class Edge, class To>
__device__ __forceinline__ void turn_rows(int rows, int per, int A, int np, bool in_place, const float2* cs, From from, Edge edge, To to) {
  const int step = pieces_at_once<P>(A, in_place);
  for (int u0 = 0; u0 < rows * per; u0 += step) {
    const int u = u0 + (int)threadIdx.x, r = u / per, w = u - r * per, h = w / A, p = w - h * A;
    const bool mine = (int)threadIdx.x < step && u < rows * per;
    if constexpr (P == PART) {
      int at = 0;
      float8_t v;
      if (mine)
        turn_piece<P, TI>(from(r, h), p, np, edge(r, h), cs + r * entries<P>(np), [&](int c, float8_t z) {
          at = c;
          v = z;
        });
      if (in_place) __syncthreads();
      if (mine) to(r, h, at, v);
    } else {
      if (mine) turn_piece<P, TI>(from(r, h), p, np, false, cs + r * entries<P>(np), [&](int c, float8_t z) { to(r, h, c, z); });
    }
  }
}

// grid (rows / a.rows, head chunks)
template <int P, int TI, int TO, bool PAST>
__global__ __launch_bounds__(kRT) void rope_kernel(const RopeArgs a) {
  extern __shared__ __align__(16) float2 cs[];
  __shared__ int pos[kRows];
  const int64_t r0 = (int64_t)blockIdx.x * a.rows;
  const int rows = (int)min((int64_t)a.rows, a.n_rows - r0);
  const int h0 = blockIdx.y * a.chunk, nh = min(a.chunk, a.n_heads - h0);
  if (threadIdx.x < rows) pos[threadIdx.x] = a.pos[r0 + threadIdx.x];
  __syncthreads();
  fill_table<P, TO>(cs, a.t, pos, rows);
  __syncthreads();
  const int np = a.t.n_pairs, A = pieces<P>(a.d), per = A * nh;
  const row_t<TI>* x = static_cast<const row_t<TI>*>(a.x);
  row_t<TO>* out = static_cast<row_t<TO>*>(a.out);
  turn_rows<P, TI>(
      rows, per, A, np, a.x == a.out, cs, [&](int r, int h) { return x + (r0 + r) * a.x_stride + (int64_t)(h0 + h) * a.d; },
      [&](int r, int h) { return (r0 + r == 0 && h0 + h == 0) || (r0 + r == a.n_rows - 1 && h0 + h == a.n_heads - 1); },
      [&](int r, int h, int c, float8_t v) { store8<TO, PAST>(out + (r0 + r) * a.out_stride + (int64_t)(h0 + h) * a.d + c, v); });
}

template <int P, int TI, int TO>
void rope_past(const RopeArgs& a, bool past, dim3 g, size_t lds, hipStream_t s) {
  if constexpr (TO != DWKV_F32) {
    if (past) {
      hipLaunchKernelGGL((rope_kernel<P, TI, TO, true>), g, dim3(kRT), lds, s, a);
      return;
    }
  }
  hipLaunchKernelGGL((rope_kernel<P, TI, TO, false>), g, dim3(kRT), lds, s, a);
}

template <int P, int TI>
void rope_out(const RopeArgs& a, int to, bool past, dim3 g, size_t lds, hipStream_t s) {
  switch (to) {
    case DWKV_F32: rope_past<P, TI, DWKV_F32>(a, past, g, lds, s); break;
    case DWKV_F16: rope_past<P, TI, DWKV_F16>(a, past, g, lds, s); break;
    default: rope_past<P, TI, DWKV_BF16>(a, past, g, lds, s); break;
  }
}

template <int P>
void rope_in(const RopeArgs& a, int from, int to, bool past, dim3 g, size_t lds, hipStream_t s) {
  switch (from) {
    case DWKV_F32: rope_out<P, DWKV_F32>(a, to, past, g, lds, s); break;
    case DWKV_F16: rope_out<P, DWKV_F16>(a, to, past, g, lds, s); break;
    default: rope_out<P, DWKV_BF16>(a, to, past, g, lds, s); break;
  }
}

// ---- append ------------------------------------------------------------------------
// Two kinds of workgroups in one launch.  The first fill pages: each takes the new rows
// that fall into 16 consecutive slots of one sequence (aligned to 16: a tile of keys,
// two blocks of values) and some of the heads of keys and values.  The others turn
// queries, a row or two each, as rope_kernel does.

// The group of 16 slots that workgroup w takes: sequence, slot / 16, and the sequence's
// rows and length.  A sequence has a group for every 16 slots that hold a new row of it.
struct Group {
  int seq, first, c0, c1, len;
};
__device__ __forceinline__ int groups_of(int rows, int len, int& first) {
  if (rows <= 0) return 0;
  first = (int)(((int64_t)len - rows) >> 4);
  return ((len - 1) >> 4) - first + 1;
}
// False past the last group.  Up to 64 sequences every wave finds it by itself.
__device__ __forceinline__ bool find_group(const AppendArgs& a, int w, Group& g) {
  __shared__ int found[5];
  __shared__ int sums[kRT / 64];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const auto upto = [&](int n) {
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(n, d);
      if (lane >= d) n += o;
    }
    return n;
  };
  if (a.batch <= 64) {
    const int b = min(lane, a.batch - 1), c0 = a.cu_new[b], c1 = a.cu_new[b + 1], len = a.len[b];
    int first = 0;
    const int n = lane < a.batch ? groups_of(c1 - c0, len, first) : 0;
    const int inc = upto(n);
    const unsigned long long here = __ballot(w < inc && w >= inc - n);
    if (!here) return false;
    const int k = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(here));
    g.seq = k;
    g.c0 = __builtin_amdgcn_readlane(c0, k);
    g.c1 = __builtin_amdgcn_readlane(c1, k);
    g.len = __builtin_amdgcn_readlane(len, k);
    g.first = __builtin_amdgcn_readlane(first, k) + w - (__builtin_amdgcn_readlane(inc, k) - __builtin_amdgcn_readlane(n, k));
    return true;
  }
  if (threadIdx.x == 0) found[0] = -1;
  int base = 0;
  for (int b0 = 0; b0 < a.batch; b0 += kRT) {
    const int b = b0 + threadIdx.x;
    int n = 0, first = 0, c0 = 0, c1 = 0, len = 0;
    if (b < a.batch) {
      c0 = a.cu_new[b];
      c1 = a.cu_new[b + 1];
      len = a.len[b];
      n = groups_of(c1 - c0, len, first);
    }
    const int inc = upto(n);
    if (lane == 63) sums[wv] = inc;
    __syncthreads();
    int before = base, total = 0;
    for (int i = 0; i < kRT / 64; ++i) {
      if (i < wv) before += sums[i];
      total += sums[i];
    }
    const int at = before + inc - n;
    if (w >= at && w < at + n) {
      found[0] = b;
      found[1] = first + (w - at);
      found[2] = c0;
      found[3] = c1;
      found[4] = len;
    }
    __syncthreads();
    base += total;
    if (base > w) break;
  }
  g = {found[0], found[1], found[2], found[3], found[4]};
  return g.seq >= 0;
}

// Where rows r0 .. r0 + rows - 1 lie in their sequences; false in `in`: behind the last start.
__device__ __forceinline__ void find_rows(const AppendArgs& a, int r0, int rows, int* place, bool* in) {
  __shared__ int before[kRows];
  const int lane = threadIdx.x & 63;
  if (!a.cu_new) {
    if (threadIdx.x < rows) {
      place[threadIdx.x] = a.len[r0 + threadIdx.x] - 1;
      in[threadIdx.x] = true;
    }
  } else if (a.batch <= 64) {
    const int b = min(lane, a.batch - 1), c1 = a.cu_new[b + 1], len = a.len[b];
    for (int j = 0; j < rows; ++j) {
      const unsigned long long after = __ballot(lane < a.batch && c1 > r0 + j);
      const int k = after ? __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(after)) : 0;
      const int at = __builtin_amdgcn_readlane(len, k) - (__builtin_amdgcn_readlane(c1, k) - (r0 + j));
      if (threadIdx.x == 0) {
        in[j] = after != 0;
        place[j] = at;
      }
    }
  } else {                               // sequences that end before the row
    if (threadIdx.x < kRows) before[threadIdx.x] = 0;
    __syncthreads();
    int n[kRows] = {};
    for (int b = threadIdx.x; b < a.batch; b += kRT) {
      const int c1 = a.cu_new[b + 1];
#pragma unroll
      for (int j = 0; j < kRows; ++j) n[j] += c1 <= r0 + j;
    }
#pragma unroll
    for (int j = 0; j < kRows; ++j) atomicAdd(&before[j], n[j]);
    __syncthreads();
    if (threadIdx.x < rows) {
      const int b = before[threadIdx.x];
      in[threadIdx.x] = b < a.batch;
      if (b < a.batch) place[threadIdx.x] = a.len[b] - (a.cu_new[b + 1] - (r0 + (int)threadIdx.x));
    }
  }
}

template <int P, int TI, int TC, bool PAST>
__device__ __forceinline__ void append_queries(const AppendArgs& a, int w, float2* cs) {
  __shared__ int pos[kRows];
  __shared__ bool in[kRows];
  const int group = w / a.q_chunks, c0 = (w - group * a.q_chunks) * a.q_chunk, nh = min(a.q_chunk, a.n_q_heads - c0);
  const int r0 = group * a.rows, rows = min(a.rows, a.n_rows - r0), np = a.t.n_pairs, d = a.d;
  find_rows(a, r0, rows, pos, in);
  __syncthreads();
  if (a.pos && threadIdx.x < rows) pos[threadIdx.x] = a.pos[r0 + threadIdx.x];
  __syncthreads();
  if (np > 0) {
    fill_table<P, TC>(cs, a.t, pos, rows);
    __syncthreads();
  }
  const int A = pieces<P>(d), per = A * nh;
  const row_t<TI>* x = static_cast<const row_t<TI>*>(a.q) + r0 * a.q_stride + (int64_t)c0 * d;
  row_t<TC>* out = static_cast<row_t<TC>*>(a.q_out) + ((int64_t)r0 * a.n_q_heads + c0) * d;
  turn_rows<P, TI>(
      rows, per, A, np, a.q == a.q_out, cs, [&](int r, int h) { return x + r * a.q_stride + (int64_t)h * d; },
      [&](int r, int h) { return (r0 + r == 0 && c0 + h == 0) || (r0 + r == a.n_rows - 1 && c0 + h == a.n_q_heads - 1); },
      [&](int r, int h, int c, float8_t z) {
        if (in[r]) store8<TC, PAST>(out + ((int64_t)r * a.n_q_heads + h) * d + c, z);
      });
}

template <int P, int TI, int TC, bool PAST>
__global__ __launch_bounds__(kRT) void append_kernel(const AppendArgs a) {
  extern __shared__ __align__(16) float2 cs[];
  __shared__ int pos[kSlots];
  if ((int)blockIdx.x >= a.n_fill) {
    append_queries<P, TI, TC, PAST>(a, blockIdx.x - a.n_fill, cs);
    return;
  }
  const int w = blockIdx.x / a.kv_chunks;
  Group g;
  int r0, end, slot0;                    // rows [r0, end) of the packed rows, r0 at slot slot0
  if (a.cu_new) {
    if (!find_group(a, w, g)) return;
    const int64_t start = (int64_t)g.len - (g.c1 - g.c0), s0 = (int64_t)g.first * 16;
    slot0 = (int)max(start, s0);
    r0 = g.c0 + (int)(slot0 - start);
    end = g.c0 + (int)(min(start + (g.c1 - g.c0), s0 + 16) - start);
    if (r0 < 0 || end <= r0 || end > a.n_rows) return;          // starts that do not fit the rows
  } else {                               // one row for each sequence
    g.seq = w;
    slot0 = a.len[g.seq] - 1;
    r0 = w;
    end = r0 + 1;
  }
  // the page of these slots: rows without one are not stored
  const int page = 16 << a.page_shift;
  if (slot0 < 0 || slot0 >= (int64_t)a.max_pages * page) return;
  const int id = a.table[(int64_t)g.seq * a.max_pages + (slot0 >> (a.page_shift + 4))];
  const int rows = end - r0, off = slot0 & 15;
  const int np = a.t.n_pairs, d = a.d;
  if (np > 0) {
    if (threadIdx.x < rows) pos[threadIdx.x] = a.pos ? a.pos[r0 + threadIdx.x] : slot0 + (int)threadIdx.x;
    __syncthreads();
    fill_table<P, TC>(cs, a.t, pos, rows);
  }
  __syncthreads();
  const int hk = a.n_kv_heads, c0 = ((int)blockIdx.x - w * a.kv_chunks) * a.kv_chunk, c1 = min(c0 + a.kv_chunk, 2 * hk);
  const int A = pieces<P>(d);
  if (id < 0 || id >= a.n_pages) return;
  const int t0 = slot0 & (page - 1) & ~15;                 // the group's place in its page
  const int64_t at = ((int64_t)id * hk * page + t0) * d;     // of KV head 0
  if (c0 < hk) {                         // keys: [d/8][16][8] of the tile
    const int k0 = c0, nh = min(c1, hk) - k0, per = rows * A;
    const row_t<TI>* x = static_cast<const row_t<TI>*>(a.k);
    row_t<TC>* tile = static_cast<row_t<TC>*>(a.k_pages) + at;
    for (int u = threadIdx.x; u < nh * per; u += kRT) {
      const int h = u / per + k0, w = u % per, p = w / rows, r = w - p * rows;
      row_t<TC>* y = tile + (int64_t)h * page * d + (off + r) * 8;
      turn_piece<P, TI>(
          x + (int64_t)(r0 + r) * a.kv_stride + (int64_t)h * d, p, np,
          (r0 + r == 0 && h == 0) || (r0 + r == a.n_rows - 1 && h == hk - 1), cs + r * entries<P>(np),
          [&](int c, float8_t v) { store8<TC, PAST>(y + c * 16, v); });
    }
  }
  if (c1 > hk) {                         // values: two blocks of [d][8], eight channels of eight tokens a piece
    const int v0 = max(c0, hk) - hk, nh = c1 - hk - v0, D8 = d / 8;
    const row_t<TI>* x = static_cast<const row_t<TI>*>(a.v);
    row_t<TC>* blocks = static_cast<row_t<TC>*>(a.v_pages) + at;
    for (int u = threadIdx.x; u < 2 * nh * D8; u += kRT) {
      const int p = u % D8, w = u / D8, h = (w >> 1) + v0, blk = w & 1;
      const int r_lo = max(0, blk * 8 - off), r_hi = min(rows, blk * 8 + 8 - off);   // rows of this block
      if (r_lo >= r_hi) continue;
      const row_t<TI>* src = x + (int64_t)(r0 + r_lo) * a.kv_stride + (int64_t)h * d + p * 8;
      row_t<TC>* y = blocks + (int64_t)h * page * d + (blk * d + p * 8) * 8;
      if (r_hi - r_lo == 8) {
        row8_t<TC> v[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) v[t] = __builtin_convertvector(load8<TI>(src + t * a.kv_stride), row8_t<TC>);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          row8_t<TC> o;
#pragma unroll
          for (int t = 0; t < 8; ++t) o[t] = v[t][c];
          *reinterpret_cast<row8_t<TC>*>(y + c * 8) = o;
        }
      } else {
        row8_t<TC> v[8];
        const int t0 = (off + r_lo) & 7, n = r_hi - r_lo;            // tokens t0 .. t0 + n - 1 of the block
#pragma unroll
        for (int t = 0; t < 8; ++t) v[t] = __builtin_convertvector(load8<TI>(src + min(t, n - 1) * a.kv_stride), row8_t<TC>);
#pragma unroll
        for (int t = 0; t < 8; ++t)
          if (t < n)
#pragma unroll
            for (int c = 0; c < 8; ++c) y[c * 8 + t0 + t] = v[t][c];
      }
    }
  }
}

template <int P, int TI, int TC>
void append_past(const AppendArgs& a, bool past, dim3 g, size_t lds, hipStream_t s) {
  if (past) hipLaunchKernelGGL((append_kernel<P, TI, TC, true>), g, dim3(kRT), lds, s, a);
  else hipLaunchKernelGGL((append_kernel<P, TI, TC, false>), g, dim3(kRT), lds, s, a);
}

template <int P, int TI>
void append_out(const AppendArgs& a, int to, bool past, dim3 g, size_t lds, hipStream_t s) {
  if (to == DWKV_F16) append_past<P, TI, DWKV_F16>(a, past, g, lds, s);
  else append_past<P, TI, DWKV_BF16>(a, past, g, lds, s);
}

template <int P>
void append_in(const AppendArgs& a, int from, int to, bool past, dim3 g, size_t lds, hipStream_t s) {
  switch (from) {
    case DWKV_F32: append_out<P, DWKV_F32>(a, to, past, g, lds, s); break;
    case DWKV_F16: append_out<P, DWKV_F16>(a, to, past, g, lds, s); break;
    default: append_out<P, DWKV_BF16>(a, to, past, g, lds, s); break;
  }
}

// Heads of a workgroup: all of them where rows alone give the chip four workgroups
// per compute unit, fewer otherwise, but a piece for each thread.
int head_chunk(int64_t groups, int rows, int heads, int d) {
  const int64_t want = (1024 + groups - 1) / groups;
  const int least = std::max(1, kRT / (rows * (d / 8)));
  return std::min(heads, std::max(least, (int)((heads + want - 1) / want)));
}

// Rows of a workgroup.  Few, so that the workgroups at work read and write in one place
// that moves on: with plain stores 16384 rows of 40 heads take 64 us with 2, 69, 72 and 74
// with 4, 8 and 16.
int rows_of(int64_t n_rows) { return n_rows >= 2048 ? kRows : 1; }

// Whether 16-bit numbers are written past the caches: more than the eight L2s hold.  (float32
// ones leave in two stores of half lines: 8192 rows of 40 heads of 128 take 67 us through the
// caches and 72 past them, of 256 in neighbouring pairs 143 and 192, of 64 37 and 32.)
bool past_caches(int64_t rows, int heads, int d) { return rows * heads * d * 2 > (32 << 20); }

}  // namespace

hipError_t launch_rope(RopeArgs a, int from, int to, hipStream_t s) {
  a.rows = rows_of(a.n_rows);
  const int64_t groups = (a.n_rows + a.rows - 1) / a.rows;
  a.chunk = head_chunk(groups, a.rows, a.n_heads, a.d);
  const bool past = past_caches(a.n_rows, a.n_heads, a.d);
  const dim3 g((unsigned)groups, (a.n_heads + a.chunk - 1) / a.chunk);
  const size_t lds = (size_t)a.rows * 2 * a.t.n_pairs * sizeof(float2);
  if (a.t.interleaved) rope_in<NEXT>(a, from, to, past, g, lds, s);
  else if (a.t.n_pairs % 8 == 0 && 2 * a.t.n_pairs == a.d) rope_in<HALF>(a, from, to, past, g, lds, s);
  else rope_in<PART>(a, from, to, past, g, lds, s);
  return hipGetLastError();
}

hipError_t launch_append(AppendArgs a, int from, int to, hipStream_t s) {
  // a sequence's n rows touch at most n groups, and at most n / 16 + 2
  const int64_t groups = a.cu_new ? std::min<int64_t>(a.n_rows, a.n_rows / 16 + 2 * (int64_t)a.batch) : a.n_rows;
  const int slots = a.cu_new ? std::min(kSlots, a.n_rows) : 1;
  a.kv_chunk = head_chunk(groups, slots, 2 * a.n_kv_heads, a.d);
  a.kv_chunks = (2 * a.n_kv_heads + a.kv_chunk - 1) / a.kv_chunk;
  a.rows = rows_of(a.n_rows);
  const int64_t q_groups = a.n_q_heads > 0 ? (a.n_rows + a.rows - 1) / a.rows : 0;
  a.q_chunk = a.q_chunks = 1;
  if (q_groups > 0) {
    a.q_chunk = head_chunk(q_groups, a.rows, a.n_q_heads, a.d);
    a.q_chunks = (a.n_q_heads + a.q_chunk - 1) / a.q_chunk;
  }
  a.n_fill = (int)(groups * a.kv_chunks);
  const bool past = past_caches(a.n_rows, a.n_q_heads + 2 * a.n_kv_heads, a.d);
  const dim3 g((unsigned)(a.n_fill + q_groups * a.q_chunks));
  const size_t lds = (size_t)std::max(slots, a.rows) * 2 * a.t.n_pairs * sizeof(float2);
  if (a.t.interleaved) append_in<NEXT>(a, from, to, past, g, lds, s);
  else if (a.t.n_pairs % 8 == 0 && 2 * a.t.n_pairs == a.d) append_in<HALF>(a, from, to, past, g, lds, s);
  else append_in<PART>(a, from, to, past, g, lds, s);
  return hipGetLastError();
}

}  // namespace dwkv
