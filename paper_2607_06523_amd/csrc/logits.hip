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

struct Rules {                           // of a row
  float rep, pres, freq, temp;
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
  if (!a.params) return {1.f, 0.f, 0.f, 1.f};
  const float* p = a.params + 4 * (int64_t)b;
  return {p[0], p[1], p[2], p[3]};
}

// How often the row's history holds each entry of [v0, v0 + a.run), and the bias of
// each: LDS words, kInPrompt set for a token of the prompt.
__device__ __forceinline__ void count(const LogitsArgs& a, int row, Row at, int v0, uint32_t* seen, float* bias) {
  const int run = min(a.run, a.vocab - v0), b = at.seq;
  for (int i = threadIdx.x; i < a.run / 4; i += kLT) {
    reinterpret_cast<uint4*>(seen)[i] = make_uint4(0, 0, 0, 0);
    if (a.bias) reinterpret_cast<float4*>(bias)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __syncthreads();
  if (a.bias) {                          // an entry listed twice adds twice, in the list's order
    const int e0 = max(a.cu_bias[b], 0), e1 = min(a.cu_bias[b + 1], a.n_bias);
    for (int e = e0; e < e1; e += kLT) {
      const int j = e + (int)threadIdx.x, i = j < e1 ? a.bias_id[j] - v0 : -1;
      bool left = i >= 0 && i < run;
      const float v = left ? a.bias[j] : 0.f;
      while (__syncthreads_or(left)) {
        if (left) atomicMax(&seen[i], ~threadIdx.x);       // the first in the list goes first
        __syncthreads();
        if (left && seen[i] == ~threadIdx.x) {
          bias[i] += v;
          left = false;
          seen[i] = 0;
        }
      }
    }
  }
  if (a.history) {
    const int n = (int)min((int64_t)max(a.history_len[b], 0), a.history_stride), m = a.prompt_len ? a.prompt_len[b] : 0;
    const int32_t* h = a.history + b * a.history_stride;
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += kLT) {
      const int t = h[i] - v0;
      if (t >= 0 && t < run) {
        if (i < m) atomicOr(&seen[t], kInPrompt);
        else atomicAdd(&seen[t], 1u);
      }
    }
  }
  if (a.cu_nodes && threadIdx.x < 64) {  // the path from node 0, itself not counted, to the row's node
    const int n = a.cu_nodes[b + 1] - at.first, lane = threadIdx.x;
    const int parent = lane < n ? a.parent[at.first + lane] : -1;
    int node = __builtin_amdgcn_readfirstlane(row - at.first);
    unsigned long long path = 0;
    while (node > 0) {
      path |= 1ull << node;
      const int up = __builtin_amdgcn_readlane(parent, node);
      node = up < node ? up : -1;
    }
    if ((path >> lane) & 1) {
      const int t = a.token[at.first + lane] - v0;
      if (t >= 0 && t < run) atomicAdd(&seen[t], 1u);
    }
  }
  __syncthreads();
}

// z of entries v .. v + 7 (v a multiple of 8 inside the run that begins at v0); past the row's end -inf.
template <int T>
__device__ __forceinline__ float8_t shaped(const LogitsArgs& a, const Rules& r, int row, int v0, int v, const uint32_t* seen,
                                           const float* bias) {
  const row_t<T>* l = static_cast<const row_t<T>*>(a.logits) + row * a.stride + v;
  float8_t z;
  if (v + 8 <= a.vocab && (reinterpret_cast<uintptr_t>(l) & 15) == 0) {
    z = load8<T>(l);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = v + i < a.vocab ? (float)l[i] : -__builtin_inff();
  }
  if (seen) {
    uint32_t c[8];
    *reinterpret_cast<uint4*>(c) = *reinterpret_cast<const uint4*>(seen + (v - v0));
    *reinterpret_cast<uint4*>(c + 4) = *reinterpret_cast<const uint4*>(seen + (v - v0) + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c[i]) {
        z[i] = z[i] > 0.f ? z[i] / r.rep : z[i] * r.rep;
        const uint32_t said = c[i] & ~kInPrompt;
        if (said) z[i] = z[i] - r.freq * (float)said - r.pres;
      }
  }
  if (a.bias) {
    const float8_t d = *reinterpret_cast<const float8_t*>(bias + (v - v0));
    z += d;
  }
  if (a.mask) {
    const uint32_t ok = reinterpret_cast<const uint8_t*>(a.mask + row * a.mask_stride)[v >> 3];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!((ok >> i) & 1)) z[i] = -__builtin_inff();
  }
  return z;
}

template <int T>
__device__ __forceinline__ void put(const LogitsArgs& a, int row, int v, float8_t x) {
  row_t<T>* o = static_cast<row_t<T>*>(a.out) + (int64_t)row * a.vocab + v;
  if (v + 8 <= a.vocab && (reinterpret_cast<uintptr_t>(o) & 15) == 0) {
    store8<T>(o, x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (v + i < a.vocab) o[i] = (row_t<T>)x[i];
  }
}

// A run's largest entry, where it is first, and the sum of exp2((z - top) scale).
__device__ __forceinline__ LogitsPart joined(LogitsPart x, LogitsPart y, float scale) {
  LogitsPart r;
  r.top = fmaxf(x.top, y.top);
  const float ref = r.top == -__builtin_inff() ? 0.f : r.top;
  r.sum = x.sum * __builtin_amdgcn_exp2f((x.top - ref) * scale) + y.sum * __builtin_amdgcn_exp2f((y.top - ref) * scale);
  r.first = x.top == r.top && (y.top != r.top || x.first < y.first) ? x.first : y.first;
  return r;
}
__device__ __forceinline__ LogitsPart wave_joined(LogitsPart p, float scale) {
  for (int d = 1; d < 64; d <<= 1) {
    LogitsPart o;
    o.top = __shfl_xor(p.top, d);
    o.sum = __shfl_xor(p.sum, d);
    o.first = __shfl_xor(p.first, d);
    // the same order in both lanes
    p = (threadIdx.x & d) ? joined(o, p, scale) : joined(p, o, scale);
  }
  return p;
}

constexpr float kLog2e = 1.44269504088896340736f;
__device__ __forceinline__ float scale_of(const Rules& r) { return r.temp > 0.f ? kLog2e / r.temp : 0.f; }

// grid (runs, rows): the logits out, or a run's part of the softmax
template <int T, int TO, bool PROBS>
__global__ __launch_bounds__(kLT) void logits_kernel(const LogitsArgs a) {
  extern __shared__ __align__(16) uint32_t lds[];
  __shared__ LogitsPart parts[kLWaves];
  const int row = blockIdx.y, v0 = blockIdx.x * a.run;
  const Row at = row_of(a, row);
  const Rules r = rules_of(a, at.seq);
  const bool counts = a.history || a.cu_nodes;
  float* bias = reinterpret_cast<float*>(lds + a.run);
  if (counts || a.bias) count(a, row, at, v0, lds, bias);
  const uint32_t* seen = counts ? lds : nullptr;
  const float scale = scale_of(r);
  LogitsPart p = {-__builtin_inff(), 0.f, a.vocab};
  for (int v = v0 + 8 * (int)threadIdx.x; v < min(v0 + a.run, a.vocab); v += kStep) {
    const float8_t z = shaped<T>(a, r, row, v0, v, seen, bias);
    if constexpr (PROBS) {
      LogitsPart q = {z[0], 0.f, v};
#pragma unroll
      for (int i = 1; i < 8; ++i)
        if (!(z[i] <= q.top)) {          // a number after NaN, too
          if (z[i] == z[i]) q.first = v + i;
          q.top = fmaxf(q.top, z[i]);
        }
      if (q.top != q.top) q.top = -__builtin_inff();
      const float ref = q.top == -__builtin_inff() ? 0.f : q.top;
#pragma unroll
      for (int i = 0; i < 8; ++i) q.sum += __builtin_amdgcn_exp2f((z[i] - ref) * scale);
      p = joined(p, q, scale);
    } else {
      put<TO>(a, row, v, z);
    }
  }
  if constexpr (PROBS) {
    p = wave_joined(p, scale);
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = p;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int i = 1; i < kLWaves; ++i) p = joined(p, parts[i], scale);
      a.part[(int64_t)row * a.n_run + blockIdx.x] = p;
    }
  }
}

// grid (runs, rows): the probabilities out
template <int T, int TO>
__global__ __launch_bounds__(kLT) void probs_kernel(const LogitsArgs a) {
  extern __shared__ __align__(16) uint32_t lds[];
  const int row = blockIdx.y, v0 = blockIdx.x * a.run;
  const Row at = row_of(a, row);
  const Rules r = rules_of(a, at.seq);
  const float scale = scale_of(r);
  LogitsPart p = {-__builtin_inff(), 0.f, a.vocab};      // every wave joins the row's parts, in one order
  for (int i = threadIdx.x & 63; i < a.n_run; i += 64) p = joined(p, a.part[(int64_t)row * a.n_run + i], scale);
  p = wave_joined(p, scale);
  const int v1 = min(v0 + a.run, a.vocab);
  if (!(r.temp > 0.f)) {
    for (int v = v0 + 8 * (int)threadIdx.x; v < v1; v += kStep) {
      float8_t x = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (v + i == p.first && p.top > -__builtin_inff()) x[i] = 1.f;
      put<TO>(a, row, v, x);
    }
    return;
  }
  const bool counts = a.history || a.cu_nodes;
  float* bias = reinterpret_cast<float*>(lds + a.run);
  if (counts || a.bias) count(a, row, at, v0, lds, bias);
  const uint32_t* seen = counts ? lds : nullptr;
  const float ref = p.top == -__builtin_inff() ? 0.f : p.top;
  const float f = p.sum == 0.f ? 0.f : 1.f / p.sum;
  for (int v = v0 + 8 * (int)threadIdx.x; v < v1; v += kStep) {
    float8_t z = shaped<T>(a, r, row, v0, v, seen, bias);
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = __builtin_amdgcn_exp2f((z[i] - ref) * scale) * f;
    put<TO>(a, row, v, z);
  }
}

template <int T, int TO>
void launch_t(const LogitsArgs& a, bool probs, size_t lds, hipStream_t s) {
  const dim3 g(a.n_run, a.n_rows);
  if (probs) {
    hipLaunchKernelGGL((logits_kernel<T, TO, true>), g, dim3(kLT), lds, s, a);
    hipLaunchKernelGGL((probs_kernel<T, TO>), g, dim3(kLT), lds, s, a);
  } else {
    hipLaunchKernelGGL((logits_kernel<T, TO, false>), g, dim3(kLT), lds, s, a);
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
