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
// compute unit.  Probabilities take a second launch that works z out again: reading
// the logits twice (2 to 4 bytes, from the last-level cache) is less than writing z and
// reading it.
#include <algorithm>

#include "entry.h"
#include "internal.h"
#include "rows_dev.h"

namespace dwkv {
namespace {

constexpr int kLT = 512;                 // threads of a workgroup
constexpr int kLWaves = kLT / 64;
constexpr int kStep = 8 * kLT;           // entries of one round
constexpr uint32_t kInPrompt = 1u << 31;
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
struct Lists {
  int hist[kIds], n, m;                  // history: ids, their number, the prompt's
  int id, e0, e1;                        // biases: this thread's id of the first kLT, their places
  float val;
  int parent, token;                     // of the tree's node of this lane
};
// Every kLT-th id from i0 on, -1 past the list's end; without branches, so that nothing waits between the loads.
__device__ __forceinline__ void fetch_ids(const int32_t* h, int i0, int n, int (&id)[kIds]) {
  if (n <= 0) {
#pragma unroll
    for (int j = 0; j < kIds; ++j) id[j] = -1;
    return;
  }
#pragma unroll
  for (int j = 0; j < kIds; ++j) id[j] = h[min(i0 + j * kLT, n - 1)];
#pragma unroll
  for (int j = 0; j < kIds; ++j) id[j] = i0 + j * kLT < n ? id[j] : -1;
}
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
  x.e0 = max(x.e0, 0);
  x.e1 = min(x.e1, a.n_bias);
  const int32_t* h = a.history + b * a.history_stride;
  fetch_ids(h, tid, x.n, x.hist);
  x.id = x.e0 + tid < x.e1 ? a.bias_id[x.e0 + tid] : -1;
  x.val = x.e0 + tid < x.e1 ? a.bias[x.e0 + tid] : 0.f;
  return x;
}

// How often the row's history holds each entry of [v0, v0 + a.run), and the bias of
// each: LDS words, kInPrompt set for a token of the prompt.
__device__ __forceinline__ void count(const LogitsArgs& a, int row, Row at, int v0, Lists& x, uint32_t* seen, float* bias) {
  const int run = min(a.run, a.vocab - v0), b = at.seq, tid = threadIdx.x;
  for (int i = tid; i < a.run / 4; i += kLT) {
    reinterpret_cast<uint4*>(seen)[i] = make_uint4(0, 0, 0, 0);
    if (a.bias) reinterpret_cast<float4*>(bias)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __syncthreads();
  for (int e = x.e0; e < x.e1;) {        // an entry listed twice adds twice, in the list's order
    const uint32_t i = (uint32_t)x.id - (uint32_t)v0;
    bool left = i < (uint32_t)run;
    while (__syncthreads_or(left)) {
      if (left) atomicMax(&seen[i], ~(uint32_t)tid);       // the first in the list goes first
      __syncthreads();
      if (left && seen[i] == ~(uint32_t)tid) {
        bias[i] += x.val;
        left = false;
        seen[i] = 0;
      }
    }
    e += kLT;
    x.id = e + tid < x.e1 ? a.bias_id[e + tid] : -1;
    x.val = e + tid < x.e1 ? a.bias[e + tid] : 0.f;
  }
  const int32_t* h = a.history + b * a.history_stride;
  for (int i0 = tid; i0 < x.n;) {
    const int mine = (int)min((int64_t)x.m - i0, (int64_t)kIds * kLT);     // the prompt's are the j with j * kLT < mine
#pragma unroll
    for (int j = 0; j < kIds; ++j) {
      const uint32_t i = (uint32_t)x.hist[j] - (uint32_t)v0;   // ids below 0 lie past every run
      if (i < (uint32_t)run) {
        if (j * kLT < mine) atomicOr(&seen[i], kInPrompt);
        else atomicAdd(&seen[i], 1u);
      }
    }
    i0 += kIds * kLT;
    if (i0 - tid >= x.n) break;
    fetch_ids(h, i0, x.n, x.hist);
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
      if (i < (uint32_t)run) atomicAdd(&seen[i], 1u);
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
template <int T, int R>
__device__ __forceinline__ void load(const LogitsArgs& a, int row, int v0, Mine<R>& x) {
  const row_t<T>* l = static_cast<const row_t<T>*>(a.logits) + row * a.stride;
  const uint8_t* mask = reinterpret_cast<const uint8_t*>(a.mask + row * a.mask_stride);
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int v = v0 + 8 * (int)threadIdx.x + j * kStep;
    x.z[j] = load8_near<T>(l, v, a.vocab);
    x.ok[j] = a.mask && v < a.vocab ? mask[v >> 3] : 0xff;
  }
}

__device__ __forceinline__ float changed(float l, bool seen, uint32_t said, const Rules& r) {
  const float z = seen ? l * (l > 0.f ? r.less : r.rep) : l;
  return said ? z - r.freq * (float)said - r.pres : z;
}

// l into z.  What the lists made of eight entries goes to the second launch as a byte
// of each: 0 untouched, 1 .. 126 how often it was said, kSeen in the prompt only;
// all ones: a bias or a larger count among them, their z are in the output.
constexpr uint32_t kSeen = 0x80;
template <bool TELL, int R>
__device__ __forceinline__ void shape(const LogitsArgs& a, const Rules& r, const uint32_t* seen, const float* bias, Mine<R>& x,
                                      uint2 (&code)[R]) {
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int at = 8 * (int)threadIdx.x + j * kStep;
    bool tell = false;
    code[j] = make_uint2(0, 0);
    if (seen) {
      uint32_t c[8];
      *reinterpret_cast<uint4*>(c) = *reinterpret_cast<const uint4*>(seen + at);
      *reinterpret_cast<uint4*>(c + 4) = *reinterpret_cast<const uint4*>(seen + at + 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t said = c[i] & ~kInPrompt;
        x.z[j][i] = changed(x.z[j][i], c[i] != 0, said, r);
        if constexpr (TELL) {
          (i < 4 ? code[j].x : code[j].y) |= (said ? said & 127 : c[i] ? kSeen : 0) << (8 * (i & 3));
          tell |= said > 126;
        }
      }
    }
    if (a.bias) {
      const float8_t d = *reinterpret_cast<const float8_t*>(bias + at);
#pragma unroll
      for (int i = 0; i < 8; ++i) tell |= !(d[i] == 0.f);
      x.z[j] += d;
    }
    if (tell) code[j] = make_uint2(0xffffffffu, 0xffffffffu);
  }
}

template <int R>
__device__ __forceinline__ void hide(Mine<R>& x) {         // what the mask does not allow
#pragma unroll
  for (int j = 0; j < R; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!((x.ok[j] >> i) & 1)) x.z[j][i] = -__builtin_inff();
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
__device__ __forceinline__ float scale_of(const Rules& r) { return r.temp > 0.f ? kLog2e / r.temp : 0.f; }
__device__ __forceinline__ float wave_max(float v) {
  for (int d = 1; d < 64; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {       // the same order in every lane
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ int wave_min(int v) {
  for (int d = 1; d < 64; d <<= 1) v = min(v, __shfl_xor(v, d));
  return v;
}

// Whether the second launch is told what the lists made of the entries, which it needs
// a float32 output for, rather than count again.
template <int TO>
constexpr bool kept = TO == DWKV_F32;

// grid (runs, rows): the logits out, or a run's part of the softmax: its largest entry,
// where that is first, and the sum of exp2((z - largest) scale)
template <int T, int TO, bool PROBS, int R>
__global__ __launch_bounds__(kLT) void logits_kernel(const LogitsArgs a) {
  extern __shared__ __align__(16) uint32_t lds[];
  __shared__ LogitsPart parts[kLWaves];
  const int row = blockIdx.y, v0 = blockIdx.x * a.run, tid = threadIdx.x;
  const Row at = row_of(a, row);
  const Rules r = rules_of(a, at.seq);
  const bool counts = a.history || a.cu_nodes, lists = counts || a.bias;
  float* bias = reinterpret_cast<float*>(lds + a.run);
  Mine<R> x;
  if (lists) {
    Lists w = fetch(a, at);
    load<T>(a, row, v0, x);
    count(a, row, at, v0, w, lds, bias);
    uint2 code[R];
    shape<PROBS && kept<TO>>(a, r, counts ? lds : nullptr, bias, x, code);
    if constexpr (PROBS && kept<TO>) {
#pragma unroll
      for (int j = 0; j < R; ++j) {
        const int v = v0 + 8 * tid + j * kStep;
        if (v < a.vocab) {
          a.code[row * a.code_stride + (v >> 3)] = code[j];
          if (code[j].x == 0xffffffffu) put8<TO>(a, row, v, x.z[j]);
        }
      }
    }
  } else {
    load<T>(a, row, v0, x);
  }
  hide(x);
  if constexpr (PROBS) {
    const float scale = scale_of(r);
    float top = -__builtin_inff(), sum = 0.f;
    int first = a.vocab;
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (x.z[j][i] > top) {
          top = x.z[j][i];
          first = v0 + 8 * tid + j * kStep + i;
        }
    const float mine = top;
    top = wave_max(top);
    if ((tid & 63) == 0) parts[tid >> 6].top = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kLWaves; ++i) top = fmaxf(top, parts[i].top);
    const float ref = top == -__builtin_inff() ? 0.f : top;
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += __builtin_amdgcn_exp2f((x.z[j][i] - ref) * scale);
    sum = wave_sum(sum);
    first = wave_min(mine == top ? first : a.vocab);
    if ((tid & 63) == 0) {
      parts[tid >> 6].sum = sum;
      parts[tid >> 6].first = first;
    }
    __syncthreads();
    if (tid == 0) {
      LogitsPart p = {top, 0.f, a.vocab};
#pragma unroll
      for (int i = 0; i < kLWaves; ++i) {
        p.sum += parts[i].sum;
        p.first = min(p.first, parts[i].first);
      }
      a.part[(int64_t)row * a.n_run + blockIdx.x] = p;
    }
  } else {
#pragma unroll
    for (int j = 0; j < R; ++j) put8<TO>(a, row, v0 + 8 * tid + j * kStep, x.z[j]);
  }
}

// grid (runs, rows): the probabilities out
template <int T, int TO, int R>
__global__ __launch_bounds__(kLT) void probs_kernel(const LogitsArgs a) {
  extern __shared__ __align__(16) uint32_t lds[];
  const int row = blockIdx.y, v0 = blockIdx.x * a.run, tid = threadIdx.x, lane = tid & 63;
  const Row at = row_of(a, row);
  const Rules r = rules_of(a, at.seq);
  const bool counts = a.history || a.cu_nodes, lists = counts || a.bias;
  const float scale = scale_of(r);
  Mine<R> x;
  Lists w;
  if (lists && !kept<TO>) w = fetch(a, at);
  uint2 code[R];
  if (lists && kept<TO>) {
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int v = v0 + 8 * tid + j * kStep;
      code[j] = v < a.vocab ? a.code[row * a.code_stride + (v >> 3)] : make_uint2(0, 0);
    }
  }
  load<T>(a, row, v0, x);
  // every wave joins the row's parts, in one order
  const LogitsPart* part = a.part + (int64_t)row * a.n_run;
  float top = -__builtin_inff(), sum = 0.f;
  for (int i = lane; i < a.n_run; i += 64) top = fmaxf(top, part[i].top);
  top = wave_max(top);
  const float ref = top == -__builtin_inff() ? 0.f : top;
  int first = a.vocab;
  for (int i = lane; i < a.n_run; i += 64) {
    const LogitsPart p = part[i];
    sum += p.sum * __builtin_amdgcn_exp2f((p.top - ref) * scale);
    if (p.top == top) first = min(first, p.first);
  }
  if (r.temp > 0.f) {
    sum = wave_sum(sum);
    if (lists) {
      if constexpr (kept<TO>) {
#pragma unroll
        for (int j = 0; j < R; ++j) {
          const int v = v0 + 8 * tid + j * kStep;
          if (code[j].x == 0xffffffffu) {
            x.z[j] = load8_near<DWKV_F32>(static_cast<const float*>(a.out) + (int64_t)row * a.vocab, v, a.vocab);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const uint32_t c = ((i < 4 ? code[j].x : code[j].y) >> (8 * (i & 3))) & 255;
              x.z[j][i] = changed(x.z[j][i], c != 0, c & kSeen ? 0 : c, r);
            }
          }
        }
      } else {
        float* bias = reinterpret_cast<float*>(lds + a.run);
        count(a, row, at, v0, w, lds, bias);
        shape<false>(a, r, counts ? lds : nullptr, bias, x, code);
      }
    }
    hide(x);
    const float f = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) x.z[j][i] = __builtin_amdgcn_exp2f((x.z[j][i] - ref) * scale) * f;
  } else {
    first = wave_min(first);
    const int one = top > -__builtin_inff() ? first - v0 - 8 * tid : -1;
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) x.z[j][i] = one == j * kStep + i ? 1.f : 0.f;
  }
#pragma unroll
  for (int j = 0; j < R; ++j) put8<TO>(a, row, v0 + 8 * tid + j * kStep, x.z[j]);
}

template <int T, int TO, int R>
void launch_r(const LogitsArgs& a, bool probs, size_t lds, hipStream_t s) {
  const dim3 g(a.n_run, a.n_rows);
  if (probs) {
    hipLaunchKernelGGL((logits_kernel<T, TO, true, R>), g, dim3(kLT), lds, s, a);
    hipLaunchKernelGGL((probs_kernel<T, TO, R>), g, dim3(kLT), kept<TO> ? 0 : lds, s, a);
  } else {
    hipLaunchKernelGGL((logits_kernel<T, TO, false, R>), g, dim3(kLT), lds, s, a);
  }
}

template <int T, int TO>
void launch_t(const LogitsArgs& a, bool probs, size_t lds, hipStream_t s) {
  switch (a.run / kStep) {
    case 1: launch_r<T, TO, 1>(a, probs, lds, s); break;
    case 2: launch_r<T, TO, 2>(a, probs, lds, s); break;
    default: launch_r<T, TO, 4>(a, probs, lds, s); break;
  }
}

template <int T>
void launch_from(const LogitsArgs& a, int to, bool probs, size_t lds, hipStream_t s) {
  switch (to) {
    case DWKV_F32: launch_t<T, DWKV_F32>(a, probs, lds, s); break;
    case DWKV_F16: launch_t<T, DWKV_F16>(a, probs, lds, s); break;
    default: launch_t<T, DWKV_BF16>(a, probs, lds, s); break;
  }
}

}  // namespace

// Runs of a row, for room in the workspace: the shortest.
int64_t logits_most_runs(int64_t vocab) { return (vocab + kStep - 1) / kStep; }

hipError_t launch_logits(LogitsArgs a, int from, int to, bool probs, hipStream_t s) {
  // 64 KB of LDS at most, so that a compute unit holds two workgroups
  a.run = kStep;
  while (a.run < (a.bias ? 2 : 4) * kStep && (int64_t)a.n_rows * ((a.vocab + 2 * a.run - 1) / (2 * a.run)) >= 512) a.run *= 2;
  a.n_run = (a.vocab + a.run - 1) / a.run;
  const size_t lds = a.bias ? 8 * (size_t)a.run : a.history || a.cu_nodes ? 4 * (size_t)a.run : 0;
  switch (from) {
    case DWKV_F32: launch_from<DWKV_F32>(a, to, probs, lds, s); break;
    case DWKV_F16: launch_from<DWKV_F16>(a, to, probs, lds, s); break;
    default: launch_from<DWKV_BF16>(a, to, probs, lds, s); break;
  }
  return hipGetLastError();
}

}  // namespace dwkv
