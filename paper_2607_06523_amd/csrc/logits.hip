// Penalties for repeated tokens, biases, grammar masks and temperature on rows of
// logits, and the probabilities they leave, gfx950.
//
// With the tokens of a row's history (its sequence's, then the path to a tree's node):
//   z = l;  a token seen: z > 0 ? z / repetition : z * repetition
//   said c > 0 times:     z = z - frequency c - presence
//   z = z + bias;  not allowed: z = -inf
//   p = softmax(z / temperature), or 1 at the first largest z
// A workgroup takes a run of a row's entries.  It counts the history's tokens that fall
// into its run in LDS (integers: the order does not matter), so no array of counts as
// wide as the vocabulary is kept, cleared or read; the price is that every run reads
// the whole history, so runs are as long as still give the chip two workgroups per
// compute unit.  Probabilities of short rows are made in one launch, a workgroup with its
// row in registers.  Else they take a second one that works z out again: reading the
// logits twice (2 to 4 bytes, from the last-level cache) is less than writing z and reading
// it.  It counts again too, or is told the counts, a byte an entry.
// 64 rows of 131072 float32 entries behind 16000 tokens take 14 and 17 us: the first by
// its arithmetic (28 instructions an entry, 6 us) after its loads, as all workgroups start
// together; the second the same and a write of 34 MB.
#include <algorithm>

#include "internal.h"
#include "rows_dev.h"

namespace dwkv {
namespace {

constexpr int kRunThreads = 512;         // of a workgroup with a run of a row
constexpr int kRowThreads = 1024;        // with a whole row
constexpr int kStep = 8 * kRunThreads;   // entries of a run's round; a run has 1, 2 or 4
constexpr int kMostWhole = 32 * kRowThreads;     // entries of a row that one workgroup takes (128 KB of LDS)
constexpr int kNowhere = 64;             // words of LDS behind a run's: what lies in another run counts there, a lane apart
constexpr int kIds = 16;                 // ids of the history that a thread has under way

struct Rules {                           // of a row; less = 1 / rep
  float rep, pres, freq, temp, less;
};

struct Row {
  int seq, first;                        // its sequence, and that one's first row
};
__device__ __forceinline__ Row row_of(const LogitsArgs& a, int row) {
  if (!a.cu_nodes) return {row, row};
  int b = 0, hi = a.batch;               // the last with cu[b] <= row
  while (hi - b > 1) {
    const int mid = (b + hi) >> 1;
    if (a.cu_nodes[mid] <= row) b = mid; else hi = mid;
  }
  return {b, a.cu_nodes[b]};
}

__device__ __forceinline__ Rules rules_of(const LogitsArgs& a, int b) {
  if (!a.params) return {1.f, 0.f, 0.f, 1.f, 1.f};
  const float* p = a.params + 4 * (int64_t)b;
  return {p[0], p[1], p[2], p[3], 1.f / p[0]};
}

// What counting reads first, all of it on its way at once: two waits in all, for the
// lengths and then for the first ids of each list.
typedef int int4_t __attribute__((ext_vector_type(4)));
struct Lists {
  int4_t hist[kIds / 4];                 // history: ids 4 tid + 4 NT j + k, 0 past the end
  int n, m;                              // their number, the prompt's
  int id, e0, e1;                        // biases: this thread's id of the first NT, their places
  float val;
  int parent, token;                     // of the tree's node of this lane
};
// Four ids of each kIds / 4 stretches of 4 NT from `base` on, 0 past the list's end.
template <int NT>
__device__ __forceinline__ void fetch_ids(const int32_t* h, int base, int n, int4_t (&id)[kIds / 4]) {
  const __amdgpu_buffer_rsrc_t list = __builtin_amdgcn_make_buffer_rsrc(const_cast<int32_t*>(h), 0, 4 * n, 0x00020000);
#pragma unroll
  for (int j = 0; j < kIds / 4; ++j)
    id[j] = __builtin_bit_cast(
        int4_t, __builtin_amdgcn_raw_buffer_load_b128(list, (int)(16u * (threadIdx.x + j * NT) + 4u * (uint32_t)base), 0, 0));
}
template <int NT>
__device__ __forceinline__ Lists fetch(const LogitsArgs& a, Row at) {
  const int b = at.seq, tid = threadIdx.x, lane = tid & 63;
  Lists x;
  x.n = a.history ? a.history_len[b] : 0;
  x.m = a.history && a.prompt_len ? a.prompt_len[b] : 0;
  x.e0 = a.bias ? a.cu_bias[b] : 0;
  x.e1 = a.bias ? a.cu_bias[b + 1] : 0;
  x.parent = x.token = -1;
  if (a.cu_nodes && lane < a.cu_nodes[b + 1] - at.first) {
    x.parent = a.parent[at.first + lane];
    x.token = a.token[at.first + lane];
  }
  x.n = (int)min((int64_t)max(x.n, 0), a.history_stride);
  x.e0 = min(max(x.e0, 0), a.n_bias);
  x.e1 = min(x.e1, a.n_bias);
  const int32_t* h = a.history + b * a.history_stride;
  fetch_ids<NT>(h, 0, x.n, x.hist);
  x.id = x.e0 + tid < x.e1 ? a.bias_id[x.e0 + tid] : -1;
  x.val = x.e0 + tid < x.e1 ? a.bias[x.e0 + tid] : 0.f;
  return x;
}

// A thread's own words of LDS, those of the entries that it has.
template <int NT, int R>
__device__ __forceinline__ void clear(uint32_t* words) {
#pragma unroll
  for (int j = 0; j < R; ++j) {
    uint4* w = reinterpret_cast<uint4*>(words + 8 * ((int)threadIdx.x + j * NT));
    w[0] = w[1] = make_uint4(0, 0, 0, 0);
  }
}

// How often the row's history holds each entry of [v0, v0 + a.run): LDS words, twice the
// times that it was said, and bit 0 for a token of the prompt.
template <int NT, int R>
__device__ __forceinline__ void count(const LogitsArgs& a, int row, Row at, int v0, Lists& x, uint32_t* seen) {
  const int run = min(a.run, a.vocab - v0), b = at.seq, tid = threadIdx.x;
  clear<NT, R>(seen);
  __syncthreads();
  const int32_t* h = a.history + b * a.history_stride;
  const uint32_t nowhere = a.run + (tid & 63);
  for (int base = 0; base < x.n;) {
#pragma unroll
    for (int j = 0; j < kIds / 4; ++j) {
      const int lo = base + 4 * NT * j, hi = lo + 4 * NT, at = lo + 4 * tid;
      uint32_t i[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) i[k] = (uint32_t)x.hist[j][k] - (uint32_t)v0;      // ids below 0 lie past every run
#pragma unroll
      for (int k = 0; k < 4; ++k) i[k] = i[k] < (uint32_t)run ? i[k] : nowhere;
      if (hi <= min(x.m, x.n)) {
#pragma unroll
        for (int k = 0; k < 4; ++k) atomicOr(&seen[i[k]], 1u);
      } else if (lo >= x.m && hi <= x.n) {
#pragma unroll
        for (int k = 0; k < 4; ++k) atomicAdd(&seen[i[k]], 2u);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (at + k < x.n) {
            if (at + k < x.m) atomicOr(&seen[i[k]], 1u);
            else atomicAdd(&seen[i[k]], 2u);
          }
      }
    }
    base += kIds * NT;
    if (base < x.n) fetch_ids<NT>(h, base, x.n, x.hist);
  }
  if (a.cu_nodes && tid < 64) {          // the path from node 0, itself not counted, to the row's node
    int node = __builtin_amdgcn_readfirstlane(row - at.first);
    unsigned long long path = 0;
    while (node > 0) {
      path |= 1ull << node;
      const int up = __builtin_amdgcn_readlane(x.parent, node);
      node = up < node ? up : -1;
    }
    if ((path >> tid) & 1) {
      const uint32_t i = (uint32_t)x.token - (uint32_t)v0;
      if (i < (uint32_t)run) atomicAdd(&seen[i], 2u);
    }
  }
  __syncthreads();
}

// Entries v .. v + 7 of a row of n, -inf past its end.
template <int T>
__device__ __forceinline__ float8_t load8_near(const row_t<T>* l, int v, int n) {
  float8_t x = -__builtin_inff();
  if (v + 8 <= n) {
    x = load8_any<T>(l + v);
  } else if (v < n) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (v + i < n) x[i] = (float)l[v + i];
  }
  return x;
}

// A row's entries of one thread: eight in each round, past the row's end -inf; and the bits of its mask.
template <int R>
struct Mine {
  float8_t z[R];
  uint32_t ok[R];
};
// The same as it comes from memory.  Nothing waits for it before open(): one past the row's last eight
// entries has those.
template <int T, int R>
struct Raw {
  typename AnyPlace<T>::eight l[R];
  uint32_t ok[R];
};
template <int T, int NT, int R>
__device__ __forceinline__ void load(const LogitsArgs& a, int row, int v0, Raw<T, R>& x) {
  const row_t<T>* l = static_cast<const row_t<T>*>(a.logits) + row * a.stride;
  const uint8_t* mask = reinterpret_cast<const uint8_t*>(a.mask + row * a.mask_stride);
  const int first = v0 + 8 * (int)threadIdx.x;
  if (a.vocab >= 8) {
#pragma unroll
    for (int j = 0; j < R; ++j) x.l[j] = *reinterpret_cast<const typename AnyPlace<T>::eight*>(l + min(first + 8 * j * NT, a.vocab - 8));
  }
  if (a.mask) {
#pragma unroll
    for (int j = 0; j < R; ++j) x.ok[j] = mask[min(first + 8 * j * NT, a.vocab - 1) >> 3];
  }
}
template <int T, int NT, int R>
__device__ __forceinline__ void open(const LogitsArgs& a, int row, int v0, const Raw<T, R>& x, Mine<R>& z) {
  const row_t<T>* l = static_cast<const row_t<T>*>(a.logits) + row * a.stride;
#pragma unroll
  for (int j = 0; j < R; ++j) {
    z.ok[j] = x.ok[j];
    z.z[j] = __builtin_convertvector(x.l[j], float8_t);
  }
  if (v0 + 8 * NT * R <= a.vocab) return;                // a run inside the row
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int v = v0 + 8 * ((int)threadIdx.x + j * NT);
    if (v + 8 > a.vocab) z.z[j] = load8_near<T>(l, v, a.vocab);
  }
}

// l of an entry with the count c, as count() leaves it.
__device__ __forceinline__ float changed(float l, uint32_t c, const Rules& r) {
  const float m = c != 0 ? (l > 0.f ? r.less : r.rep) : 1.f;
  const float off = c > 1 ? __builtin_fmaf(r.freq, (float)(c >> 1), r.pres) : 0.f;
  return __builtin_fmaf(l, m, -off);
}

// The low bytes of four words.
__device__ __forceinline__ uint32_t bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}

// l into z by the counts.  With a.tell the second launch is told what the lists made of
// eight entries as a byte of each, its count up to 253; all ones: a bias or a larger
// count among them, their z are in the output.
template <bool TELL, int NT, int R>
__device__ __forceinline__ void shape(const LogitsArgs& a, const Rules& r, const uint32_t* seen, Mine<R>& x, uint2 (&code)[R]) {
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int at = 8 * ((int)threadIdx.x + j * NT);
    uint32_t c[8];
    *reinterpret_cast<uint4*>(c) = *reinterpret_cast<const uint4*>(seen + at);
    *reinterpret_cast<uint4*>(c + 4) = *reinterpret_cast<const uint4*>(seen + at + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) x.z[j][i] = changed(x.z[j][i], c[i], r);
    if (TELL && a.tell) {
      code[j] = make_uint2(bytes(c[0], c[1], c[2], c[3]), bytes(c[4], c[5], c[6], c[7]));
      if (max(max(max(c[0], c[1]), max(c[2], c[3])), max(max(c[4], c[5]), max(c[6], c[7]))) > 253)
        code[j] = make_uint2(0xffffffffu, 0xffffffffu);
    }
  }
}

// The row's biases to z, by way of the words that held the counts.  An entry listed
// twice adds twice, in the list's order: the first of those left has the word, the
// others go on when it has added.
template <bool TELL, int NT, int R>
__device__ __forceinline__ void add_bias(const LogitsArgs& a, int v0, Lists& x, uint32_t* words, Mine<R>& z, uint2 (&code)[R]) {
  __shared__ int again;
  const int run = min(a.run, a.vocab - v0), tid = threadIdx.x;
  clear<NT, R>(words);                   // own ones: the counts in them have been read
  __syncthreads();
  bool empty = true;                     // every word
  for (int e = x.e0; e < x.e1;) {
    const uint32_t i = (uint32_t)x.id - (uint32_t)v0;
    bool left = i < (uint32_t)run;
    for (;;) {
      float sum = 0.f;
      if (!empty) {
        if (left) sum = __builtin_bit_cast(float, words[i]);
        __syncthreads();
        if (left) words[i] = 0;
        __syncthreads();
      }
      if (tid == 0) again = 0;
      if (left) atomicMax(&words[i], ~(uint32_t)tid);
      __syncthreads();
      const bool mine = left && words[i] == ~(uint32_t)tid;
      left = left && !mine;
      if (left) again = 1;
      __syncthreads();
      if (mine) words[i] = __builtin_bit_cast(uint32_t, sum + x.val);
      const bool more = again;
      __syncthreads();
      empty = false;
      if (!more) break;
    }
    e += NT;
    x.id = e + tid < x.e1 ? a.bias_id[e + tid] : -1;
    x.val = e + tid < x.e1 ? a.bias[e + tid] : 0.f;
  }
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const float8_t d = *reinterpret_cast<const float8_t*>(words + 8 * (tid + j * NT));
    z.z[j] += d;
    if (TELL && a.tell) {
      uint32_t any = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) any |= __builtin_bit_cast(uint32_t, (float)d[i]);
      if (any != 0) code[j] = make_uint2(0xffffffffu, 0xffffffffu);
    }
  }
}

template <int R>
__device__ __forceinline__ void hide(const LogitsArgs& a, Mine<R>& x) {     // what the mask does not allow
  if (!a.mask) return;
#pragma unroll
  for (int j = 0; j < R; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t keep = (uint32_t)((int32_t)(x.ok[j] << (31 - i)) >> 31);
      x.z[j][i] = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, (float)x.z[j][i]) & keep) | (0xff800000u & ~keep));
    }
}

// Eight entries of the output from v on.
template <int T>
__device__ __forceinline__ void put8(const LogitsArgs& a, int row, int v, float8_t x) {
  row_t<T>* o = static_cast<row_t<T>*>(a.out) + (int64_t)row * a.vocab;
  if (v + 8 <= a.vocab) {
    store8_any<T>(o + v, x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (v + i < a.vocab) o[v + i] = (row_t<T>)x[i];
  }
}

constexpr float kLog2e = 1.44269504088896340736f;
// Entries are weighed by exp2 of half their distance to the largest (two finite ones may lie further
// apart than float32 reaches) times twice the inverse of the temperature.  That is neither infinite
// nor 0, so that 0 and -inf times it stay what they are: a temperature of +inf makes what is
// allowed even (off by 2^-21 between float32's lowest and highest numbers), the smallest one leaves the
// largest entries.
__device__ __forceinline__ float scale_of(const Rules& r) {
  return r.temp > 0.f ? fminf(fmaxf(2.f * kLog2e / r.temp, 0x1p-149f), 0x1.fffffep127f) : 0.f;
}
__device__ __forceinline__ float weight(float z, float half_ref, float scale) {
  return __builtin_amdgcn_exp2f(__builtin_fmaf(z, 0.5f, -half_ref) * scale);
}
// op over a wave's lanes, which all get it: within rows of 16 by rotation, then rows and halves
// against each other.  Both sides of each step are the same two numbers: one order in every lane.
template <int N>
__device__ __forceinline__ int rotated(int v) {
  return __builtin_amdgcn_update_dpp(0, v, 0x120 + N, 0xf, 0xf, true);
}
template <class V, class Op>
__device__ __forceinline__ V wave_all(V v, Op op) {
  const auto bits = [](V x) { return __builtin_bit_cast(int, x); };
  const auto from = [](int x) { return __builtin_bit_cast(V, x); };
  v = op(v, from(rotated<8>(bits(v))));
  v = op(v, from(rotated<4>(bits(v))));
  v = op(v, from(rotated<2>(bits(v))));
  v = op(v, from(rotated<1>(bits(v))));
  const auto rows = __builtin_amdgcn_permlane16_swap((uint32_t)bits(v), (uint32_t)bits(v), false, false);
  v = op(from((int)rows[0]), from((int)rows[1]));
  const auto halves = __builtin_amdgcn_permlane32_swap((uint32_t)bits(v), (uint32_t)bits(v), false, false);
  return op(from((int)halves[0]), from((int)halves[1]));
}
__device__ __forceinline__ float wave_max(float v) {
  return wave_all(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_sum(float v) {
  return wave_all(v, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ int wave_min(int v) {
  return wave_all(v, [](int a, int b) { return min(a, b); });
}

// Whether the second launch may be told what the lists made of the entries, which it
// needs a float32 output for, rather than count again.
template <int TO>
constexpr bool tells = TO == DWKV_F32;

// What the first launch makes of a run: its logits; its part of the softmax (the largest
// entry, the sum of exp2 of the distances to it, and for a greedy row where it is
// first); or, where a run is a whole row, its probabilities.
enum Makes { LOGITS, PART, WHOLE };

// The weights of this thread's entries, and their sum.
template <int R>
__device__ __forceinline__ float weights(const Mine<R>& x, float top, float scale, float8_t (&e)[R]) {
  const float ref = top == -__builtin_inff() ? 0.f : 0.5f * top;
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < R; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      e[j][i] = weight(x.z[j][i], ref, scale);
      sum += e[j][i];
    }
  return sum;
}

// grid (runs, rows)
template <int T, int TO, Makes M, int R>
__global__ __launch_bounds__(M == WHOLE ? kRowThreads : kRunThreads) void logits_kernel(const LogitsArgs a) {
  constexpr int NT = M == WHOLE ? kRowThreads : kRunThreads, NW = NT / 64;
  extern __shared__ __align__(16) uint32_t lds[];
  __shared__ LogitsPart parts[NW];
  const int row = blockIdx.y, v0 = blockIdx.x * a.run, tid = threadIdx.x;
  Raw<T, R> raw;
  Mine<R> x;
  load<T, NT>(a, row, v0, raw);          // on its way while the lists are found and counted
  const Row at = row_of(a, row);
  const Rules r = rules_of(a, at.seq);
  const bool counts = a.history || a.cu_nodes;
  Lists w;
  if (counts || a.bias) w = fetch<NT>(a, at);
  if (counts) count<NT, R>(a, row, at, v0, w, lds);
  open<T, NT>(a, row, v0, raw, x);
  constexpr bool TELL = M == PART && tells<TO>;
  uint2 code[R] = {};
  if (counts) shape<TELL, NT>(a, r, lds, x, code);
  if (a.bias) add_bias<TELL, NT>(a, v0, w, lds, x, code);
  if (TELL && a.tell) {
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int v = v0 + 8 * (tid + j * NT);
      if (v < a.vocab) {
        a.code[row * a.code_stride + (v >> 3)] = code[j];
        if (code[j].x == 0xffffffffu) put8<TO>(a, row, v, x.z[j]);
      }
    }
  }
  hide(a, x);
  if constexpr (M == LOGITS) {
#pragma unroll
    for (int j = 0; j < R; ++j) put8<TO>(a, row, v0 + 8 * (tid + j * NT), x.z[j]);
    return;
  }
  const float scale = scale_of(r);
  float top = -__builtin_inff();
#pragma unroll
  for (int j = 0; j < R; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, x.z[j][i]);
  top = wave_max(top);
  if ((tid & 63) == 0) parts[tid >> 6].top = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NW; ++i) top = fmaxf(top, parts[i].top);
  float8_t e[R];
  float sum = 0.f;
  int first = a.vocab;
  if (r.temp > 0.f) {
    sum = wave_sum(weights(x, top, scale, e));
  } else {
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (x.z[j][i] == top) first = min(first, v0 + 8 * (tid + j * NT) + i);
    first = wave_min(first);
  }
  if ((tid & 63) == 0) {
    parts[tid >> 6].sum = sum;
    parts[tid >> 6].first = first;
  }
  __syncthreads();
  sum = 0.f;
  first = a.vocab;
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    sum += parts[i].sum;
    first = min(first, parts[i].first);
  }
  if constexpr (M == PART) {
    if (tid == 0) a.part[(int64_t)row * a.n_run + blockIdx.x] = {top, sum, first};
  } else {
    const float f = sum == 0.f ? 0.f : 1.f / sum;
    const int one = top > -__builtin_inff() ? first - 8 * tid : -1;
#pragma unroll
    for (int j = 0; j < R; ++j) {
#pragma unroll
      for (int i = 0; i < 8; ++i) e[j][i] = r.temp > 0.f ? e[j][i] * f : one == 8 * j * NT + i ? 1.f : 0.f;
      put8<TO>(a, row, 8 * (tid + j * NT), e[j]);
    }
  }
}

// grid (runs, rows): the probabilities out
template <int T, int TO, int R>
__global__ __launch_bounds__(kRunThreads) void probs_kernel(const LogitsArgs a) {
  constexpr int NT = kRunThreads;
  extern __shared__ __align__(16) uint32_t lds[];
  const int row = blockIdx.y, v0 = blockIdx.x * a.run, tid = threadIdx.x, lane = tid & 63;
  const Row at = row_of(a, row);
  const Rules r = rules_of(a, at.seq);
  const bool counts = a.history || a.cu_nodes, told = tells<TO> && a.tell;
  const float scale = scale_of(r);
  // every wave joins the row's parts, in one order
  const LogitsPart* part = a.part + (int64_t)row * a.n_run;
  if (!(r.temp > 0.f)) {
    float top = -__builtin_inff();
    int first = a.vocab;
    for (int i = lane; i < a.n_run; i += 64) top = fmaxf(top, part[i].top);
    top = wave_max(top);
    for (int i = lane; i < a.n_run; i += 64)
      if (part[i].top == top) first = min(first, part[i].first);
    first = wave_min(first);
    const int one = top > -__builtin_inff() ? first - v0 - 8 * tid : -1;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      float8_t e;
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = one == 8 * j * NT + i ? 1.f : 0.f;
      put8<TO>(a, row, v0 + 8 * (tid + j * NT), e);
    }
    return;
  }
  Raw<T, R> raw;
  Mine<R> x;
  Lists w;
  uint2 code[R];
  if (told) {
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int v = v0 + 8 * (tid + j * NT);
      code[j] = v < a.vocab ? a.code[row * a.code_stride + (v >> 3)] : make_uint2(0, 0);
    }
  } else if (counts || a.bias) {
    w = fetch<NT>(a, at);
  }
  load<T, NT>(a, row, v0, raw);
  float top = -__builtin_inff(), sum = 0.f;
  for (int i = lane; i < a.n_run; i += 64) top = fmaxf(top, part[i].top);
  top = wave_max(top);
  const float ref = top == -__builtin_inff() ? 0.f : 0.5f * top;
  for (int i = lane; i < a.n_run; i += 64) sum += part[i].sum * weight(part[i].top, ref, scale);
  sum = wave_sum(sum);
  if (!told && counts) count<NT, R>(a, row, at, v0, w, lds);
  open<T, NT>(a, row, v0, raw, x);
  if (told) {
#pragma unroll
    for (int j = 0; j < R; ++j) {
      if (code[j].x == 0xffffffffu) {
        x.z[j] = load8_near<DWKV_F32>(static_cast<const float*>(a.out) + (int64_t)row * a.vocab, v0 + 8 * (tid + j * NT), a.vocab);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t c = ((i < 4 ? code[j].x : code[j].y) >> (8 * (i & 3))) & 255;
          if (__any(c != 0)) x.z[j][i] = changed(x.z[j][i], c, r);     // few entries are in a list: often a wave has none of its 64
        }
      }
    }
  } else {
    if (counts) shape<false, NT>(a, r, lds, x, code);
    if (a.bias) add_bias<false, NT>(a, v0, w, lds, x, code);
  }
  hide(a, x);
  float8_t e[R];
  weights(x, top, scale, e);
  const float f = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int j = 0; j < R; ++j) put8<TO>(a, row, v0 + 8 * (tid + j * NT), e[j] * f);
}

template <int T, int TO, Makes M, int R>
hipError_t launch_one(const LogitsArgs& a, size_t lds, hipStream_t s) {
  if (lds > 64 * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)logits_kernel<T, TO, M, R>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (M == PART && e == hipSuccess)
      e = hipFuncSetAttribute((const void*)probs_kernel<T, TO, R>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  const dim3 g(a.n_run, a.n_rows);
  hipLaunchKernelGGL((logits_kernel<T, TO, M, R>), g, dim3(M == WHOLE ? kRowThreads : kRunThreads), lds, s, a);
  if constexpr (M == PART) hipLaunchKernelGGL((probs_kernel<T, TO, R>), g, dim3(kRunThreads), a.tell ? 0 : lds, s, a);
  return hipGetLastError();
}

template <int T, int TO, Makes M>
hipError_t launch_r(const LogitsArgs& a, size_t lds, hipStream_t s) {
  switch (a.run / (8 * (M == WHOLE ? kRowThreads : kRunThreads))) {
    case 1: return launch_one<T, TO, M, 1>(a, lds, s);
    case 2: return launch_one<T, TO, M, 2>(a, lds, s);
    default: return launch_one<T, TO, M, 4>(a, lds, s);
  }
}

template <int T, int TO>
hipError_t launch_t(const LogitsArgs& a, bool probs, size_t lds, hipStream_t s) {
  if (!probs) return launch_r<T, TO, LOGITS>(a, lds, s);
  return a.whole ? launch_r<T, TO, WHOLE>(a, lds, s) : launch_r<T, TO, PART>(a, lds, s);
}

template <int T>
hipError_t launch_from(const LogitsArgs& a, int to, bool probs, size_t lds, hipStream_t s) {
  switch (to) {
    case DWKV_F32: return launch_t<T, DWKV_F32>(a, probs, lds, s);
    case DWKV_F16: return launch_t<T, DWKV_F16>(a, probs, lds, s);
    default: return launch_t<T, DWKV_BF16>(a, probs, lds, s);
  }
}

}  // namespace

// Runs of a row, for room in the workspace: the shortest.
int64_t logits_most_runs(int64_t vocab) { return (vocab + kStep - 1) / kStep; }

hipError_t launch_logits(LogitsArgs a, int from, int to, bool probs, hipStream_t s) {
  const bool lists = a.bias || a.history || a.cu_nodes;
  a.run = kStep;
  // One launch instead of two: 1, 64 and 256 rows of 16000 entries behind 2000 tokens take
  // 7.9, 8.7 and 12 us in it and 8.1, 9.7 and 17 in two; of 32000, where one workgroup is
  // slow, 10.9, 12.6 and 18 against 8.3, 12.1 and 26.
  a.whole = probs && a.vocab <= (a.n_rows >= 128 ? kMostWhole : kMostWhole / 2);
  if (a.whole) {
    for (a.run = 8 * kRowThreads; a.run < a.vocab;) a.run *= 2;
  } else {
    // 64 KB of LDS at most and a little, so that a compute unit holds two workgroups
    while (a.run < 4 * kStep && (int64_t)a.n_rows * ((a.vocab + 2 * a.run - 1) / (2 * a.run)) >= 512) a.run *= 2;
  }
  a.n_run = (a.vocab + a.run - 1) / a.run;
  // A byte an entry written and read, or the lists counted again: 1 row of 131072, 16 of
  // 131072 and 48 of 131072 (runs of 4096 and 8192) 8.1, 11.4 and 22.2 us told, 9.5, 12.9 and
  // 22.9 not.  In the longest runs 64 of 131072 behind 8000 tokens 28.6 and 27.1, behind 16000, 32000 and
  // 64000 32.7, 37.4 and 44.3 told, 35.5, 44.9 and 59.4 not.  The host knows the lists' room, not
  // their lengths: 500 tokens where there is room for 32768 take 25.0 told and 24.8 not, 256 such
  // rows 80 and 78.
  a.tell = probs && !a.whole && lists && to == DWKV_F32 && (a.run < 4 * kStep || a.history_stride > a.run);
  const size_t lds = lists ? (size_t)4 * (a.run + kNowhere) : 0;
  switch (from) {
    case DWKV_F32: return launch_from<DWKV_F32>(a, to, probs, lds, s);
    case DWKV_F16: return launch_from<DWKV_F16>(a, to, probs, lds, s);
    default: return launch_from<DWKV_BF16>(a, to, probs, lds, s);
  }
}

}  // namespace dwkv
