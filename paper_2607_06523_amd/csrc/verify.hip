// Verification of drafted tokens against the target's probabilities, gfx950.
//
// Children drawn independently from q and rejected one after another leave
// max(max(p - c q, 0) / Z - q, 0) = max(p - (c + Z) q, 0) / Z of the target, so
// what k rejections leave is r_k = max(p - c_k q, 0) with one number
// c_{k+1} = c_k + Z_k, Z_k = sum r_k, and whether a child stands depends on its
// parent's row and its place among the children alone, not on the walk:
//  * verify_z_kernel, for k = 1 .. max_children - 1 (with a draft): Z_k of every
//    row whose first k children are all rejected and that has one more
//  * verify_sum_kernel: every workgroup walks the tree (a lane per node, its
//    numbers gathered at once), then sums r of the last row over its chunk
//  * verify_next_kernel: finds the chunk and then the entry the next token's
//    number falls into.
// Bound by latency: a call reads few rows.  A sampled tree of 64 nodes and 4 children
// over 131072 entries takes 24 us in five launches (3 x 5.4, 6.9 and 3.9 us), a batch
// of 16 trees of the most likely tokens 14.5 in two (6.7 and 5.1); a chain's two take
// 5.1 and 3.6, less than the host needs to call them.  Chunks of 4096 entries for Z
// (one row of the fp32 pair is 1 MB) and 2048 for the sums give it 32 and 64 workgroups
// a row.  Sums are float64 in a fixed order
// and nothing is contracted, so borders fall where the definition puts them.
#include "entry.h"
#include "internal.h"

#pragma clang fp contract(off)

namespace dwkv {
namespace {

constexpr int kVT = 256;                 // threads of a workgroup
constexpr int MN = DWKV_MAX_TREE_NODES;  // one wave holds a sequence's nodes

// What is not positive and finite counts as 0.
__device__ __forceinline__ double usable(float v) { return v > 0.f && v < __builtin_inff() ? (double)v : 0.0; }

template <int PT>
__device__ __forceinline__ double prob(const void* p, int64_t i) {
  if constexpr (PT == DWKV_F32) return usable(static_cast<const float*>(p)[i]);
  const uint16_t b = static_cast<const uint16_t*>(p)[i];
  return usable(PT == DWKV_F16 ? half_bits_to_float(b) : bf16_bits_to_float(b));
}

// A sequence's nodes, one per lane: parent row (inside the sequence, -1: none),
// and the numbers of its test.
struct Node {
  int parent;
  double u, p, q;
};

__device__ __forceinline__ int parent_of(const VerifyArgs& a, int n0, int n, int lane) {
  const int p = lane > 0 && lane < n ? a.parent[n0 + lane] : -1;
  return p >= 0 && p < lane ? p : -1;
}

template <int PT>
__device__ __forceinline__ Node load_node(const VerifyArgs& a, int n0, int lane, int parent, int token) {
  Node d{parent, 0.0, 0.0, 0.0};
  if (parent >= 0) {
    d.u = (double)a.u[n0 + lane];
    if (token >= 0 && token < a.vocab) {
      d.p = prob<PT>(a.target, (int64_t)(n0 + parent) * a.vocab + token);
      if (a.draft) d.q = prob<PT>(a.draft, (int64_t)(n0 + parent) * a.vocab + token);
    }
  }
  return d;
}

// Z_k of row `row` (k >= 1): a lane per chunk in turn, then the lanes' sums, in a fixed order.
__device__ __forceinline__ double row_z(const VerifyArgs& a, int row, int k, int lane) {
  const double* z = a.z + ((int64_t)row * (a.max_children - 1) + (k - 1)) * a.zblk;
  double s = 0.0;
  for (int i = lane; i < a.zblk; i += 64) s += z[i];
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  return s;
}

// Tests the children of node `at` in index order, at most `limit` of them; the one
// that stands, or -1.  k counts the rejected, c is theirs, out their distinct
// tokens' nodes (without a draft; token: the lane's token).
__device__ __forceinline__ int test_children(const VerifyArgs& a, int n0, const Node& d, int token, int at, int limit, int lane, int& k,
                                             double& c, unsigned long long& out) {
  unsigned long long kids = __ballot(d.parent == at);
  double Z = 1.0;
  c = 0.0;
  k = 0;
  out = 0;
  while (kids && k < limit) {
    const int j = __ffsll(kids) - 1;
    kids &= kids - 1;
    const double u = __shfl(d.u, j), p = __shfl(d.p, j), q = __shfl(d.q, j);
    if (a.draft) {
      const double r = fmax(p - c * q, 0.0);
      if (u * q * Z < r) return j;
      c += Z;
      ++k;
      if (kids && k < limit) Z = row_z(a, n0 + at, k, lane);
    } else {
      // a token rejected before is left out already
      const bool again = (__ballot(token == __shfl(token, j)) & out) != 0;
      const double r = again ? 0.0 : p;
      if (u * Z < r) return j;
      Z -= r;
      ++k;
      if (!again) out |= 1ull << j;
    }
  }
  return -1;
}

__device__ __forceinline__ double block_sum(double v, double* red) {   // to every thread, fixed order
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
  for (int i = 0; i < kVT / 64; ++i) s += red[i];
  __syncthreads();
  return s;
}

// grid (zblk, N): Z_k of the row's chunk, where the walk may need it
template <int PT>
__global__ __launch_bounds__(kVT) void verify_z_kernel(const VerifyArgs a, int k) {
  __shared__ double red[kVT / 64];
  const int row = blockIdx.y, lane = threadIdx.x & 63;
  int b = 0, hi = a.batch;               // the row's sequence: the last with cu[b] <= row
  while (hi - b > 1) {
    const int mid = (b + hi) >> 1;
    if (a.cu_nodes[mid] <= row) b = mid; else hi = mid;
  }
  const int n0 = a.cu_nodes[b], n = a.cu_nodes[b + 1] - n0;
  // every wave decides for itself
  const int parent = parent_of(a, n0, n, lane);
  if (min(__popcll(__ballot(parent == row - n0)), a.max_children) <= k) return;
  const int token = lane < n ? a.token[n0 + lane] : -1;
  const Node d = load_node<PT>(a, n0, lane, parent, token);
  int tried;
  double c;
  unsigned long long out;
  if (test_children(a, n0, d, token, row - n0, k, lane, tried, c, out) >= 0) return;
  const int v0 = blockIdx.x * kVerifyZChunk, v1 = min(v0 + kVerifyZChunk, a.vocab);
  const int64_t at = (int64_t)row * a.vocab;
  double s = 0.0;
#pragma unroll 8
  for (int v = v0 + threadIdx.x; v < v1; v += kVT) s += fmax(prob<PT>(a.target, at + v) - c * prob<PT>(a.draft, at + v), 0.0);
  s = block_sum(s, red);
  if (threadIdx.x == 0) a.z[((int64_t)row * (a.max_children - 1) + (k - 1)) * a.zblk + blockIdx.x] = s;
}

// Entries v .. v + 7 of a row, past its end 0; 16 bytes at a time where the row's
// place allows it (v is a multiple of 8).
template <int PT>
__device__ __forceinline__ void load8(const void* p, int64_t row, int v, int vocab, double (&x)[8]) {
  constexpr int E = PT == DWKV_F32 ? 4 : 8;            // entries in 16 bytes
  const int64_t at = row * vocab + v;
  if (v + 8 <= vocab && (reinterpret_cast<uintptr_t>(p) / (16 / E) + at) % E == 0) {
#pragma unroll
    for (int i = 0; i < 8; i += E) {
      const uint4 w = *reinterpret_cast<const uint4*>(static_cast<const char*>(p) + (at + i) * (16 / E));
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int k = 0; k < E; ++k) {
        if constexpr (PT == DWKV_F32) {
          x[i + k] = usable(__builtin_bit_cast(float, u[k]));
        } else {
          const uint16_t h = (uint16_t)(u[k >> 1] >> (16 * (k & 1)));
          x[i + k] = usable(PT == DWKV_F16 ? half_bits_to_float(h) : bf16_bits_to_float(h));
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = v + i < vocab ? prob<PT>(p, at + i) : 0.0;
  }
}

// r of entries v .. v + 7 of the last row, past the end 0.
template <int PT>
__device__ __forceinline__ void left8(const VerifyArgs& a, const VerifyEnd& e, int64_t row, int v, double (&r)[8]) {
  load8<PT>(a.target, row, v, a.vocab, r);
  if (e.c > 0.0) {
    double q[8];
    load8<PT>(a.draft, row, v, a.vocab, q);
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = fmax(r[i] - e.c * q[i], 0.0);
  }
  for (int j = 0; j < e.n_out; ++j) {
    const int x = e.out[j] - v;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (x == i) r[i] = 0.0;
  }
}

// What the threads before this one hold of `mine`, and the sum of all, in a fixed order.
__device__ __forceinline__ double block_scan(double mine, double* red, double& total) {
  double inc = mine;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  for (int d = 1; d < 64; d <<= 1) {
    const double o = __shfl_up(inc, d);
    if (lane >= d) inc += o;
  }
  if (lane == 63) red[wv] = inc;
  double before = __shfl_up(inc, 1);
  if (lane == 0) before = 0.0;
  __syncthreads();
  total = 0.0;
  for (int i = 0; i < kVT / 64; ++i) {
    if (i == wv) before += total;
    total += red[i];
  }
  __syncthreads();
  return before;
}

// The running sum before this thread's eight entries of a chunk, and the
// chunk's sum: the same additions in both kernels.
__device__ __forceinline__ double chunk_scan(const double (&r)[8], double* red, double& total) {
  double mine = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) mine += r[i];
  return block_scan(mine, red, total);
}

// grid (nblk, B)
template <int PT>
__global__ __launch_bounds__(kVT) void verify_sum_kernel(const VerifyArgs a) {
  __shared__ double red[kVT / 64];
  __shared__ VerifyEnd e;
  const int b = blockIdx.y, lane = threadIdx.x & 63;
  const int n0 = a.cu_nodes[b], n = a.cu_nodes[b + 1] - n0;
  const bool writes = blockIdx.x == 0;
  if (n <= 0) {
    if (writes && threadIdx.x == 0) {
      a.n_kept[b] = 0;
      a.end[b].node = -1;
    }
    return;
  }
  if (threadIdx.x < 64) {
    const int token = lane < n ? a.token[n0 + lane] : -1;
    const Node d = load_node<PT>(a, n0, lane, parent_of(a, n0, n, lane), token);
    int at = 0, kept = 1, k;
    int path = lane == 0 ? 0 : -1;
    double c;
    unsigned long long out;
    for (;;) {
      const int j = test_children(a, n0, d, token, at, a.max_children, lane, k, c, out);
      if (j < 0) break;
      at = j;
      if (lane == kept) path = j;
      ++kept;
    }
    if (lane == 0) {
      e.node = at;
      e.c = c;
      e.n_out = __popcll(out);
    }
    if ((out >> lane) & 1) e.out[__popcll(out & ((1ull << lane) - 1))] = token;
    if (writes) {
      if (lane < n) a.path[n0 + lane] = path;
      if (lane == 0) a.n_kept[b] = kept;
    }
  }
  __syncthreads();
  static_assert(sizeof(VerifyEnd) % 4 == 0 && sizeof(VerifyEnd) / 4 <= kVT, "copied a word per thread");
  if (writes && threadIdx.x < sizeof(VerifyEnd) / 4)
    reinterpret_cast<uint32_t*>(&a.end[b])[threadIdx.x] = reinterpret_cast<const uint32_t*>(&e)[threadIdx.x];
  double r[8], total;
  left8<PT>(a, e, n0 + e.node, blockIdx.x * kVerifyChunk + 8 * threadIdx.x, r);
  chunk_scan(r, red, total);
  if (threadIdx.x == 0) a.sum[(int64_t)b * a.nblk + blockIdx.x] = total;
}

// The lowest thread's first place that passes the number or, when rounding lets
// none pass, the highest thread's last place with something left; and what
// came before it.  Every thread gets the answer.
struct Pick {
  int place[2][kVT / 64];
  double before[2][kVT / 64];
};
__device__ __forceinline__ int pick(Pick& sm, int first, double at_first, int last, double at_last, double& before) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const unsigned long long f = __ballot(first >= 0), l = __ballot(last >= 0);
  if (lane == (f ? __ffsll(f) - 1 : 0)) {
    sm.place[0][wv] = first;
    sm.before[0][wv] = at_first;
  }
  if (lane == (l ? 63 - __clzll(l) : 0)) {
    sm.place[1][wv] = last;
    sm.before[1][wv] = at_last;
  }
  __syncthreads();
  int at = -1;
  for (int i = kVT / 64 - 1; i >= 0; --i)
    if (sm.place[0][i] >= 0) at = sm.place[0][i], before = sm.before[0][i];
  if (at < 0)
    for (int i = 0; i < kVT / 64; ++i)
      if (sm.place[1][i] >= 0) at = sm.place[1][i], before = sm.before[1][i];
  __syncthreads();
  return at;
}

// grid (B)
template <int PT>
__global__ __launch_bounds__(kVT) void verify_next_kernel(const VerifyArgs a) {
  __shared__ double red[kVT / 64];
  __shared__ VerifyEnd e;
  __shared__ Pick pk;
  __shared__ unsigned long long best;
  const int b = blockIdx.x;
  const double u = (double)a.u_next[b];
  const int n0 = a.cu_nodes[b];
  if (threadIdx.x < sizeof(VerifyEnd) / 4)
    reinterpret_cast<uint32_t*>(&e)[threadIdx.x] = reinterpret_cast<const uint32_t*>(&a.end[b])[threadIdx.x];
  // the chunks' sums, a run of them per thread
  const double* sums = a.sum + (int64_t)b * a.nblk;
  const int per = (a.nblk + kVT - 1) / kVT, c0 = min((int)threadIdx.x * per, a.nblk), c1 = min(c0 + per, a.nblk);
  double mine = 0.0, total;
  for (int i = c0; i < c1; ++i) mine += sums[i];
  double run = block_scan(mine, red, total);
  if (e.node < 0) {                      // no nodes, and nothing in the sums
    if (threadIdx.x == 0) a.next[b] = -1;
    return;
  }
  const int64_t row = n0 + e.node;
  if (!(total > 0.0)) {                  // nothing left: the first largest p
    if (threadIdx.x == 0) best = 0;
    __syncthreads();
    unsigned long long top = 0;
    for (int v = threadIdx.x; v < a.vocab; v += kVT) {
      const float p = (float)prob<PT>(a.target, row * a.vocab + v);
      const unsigned long long key = ((unsigned long long)__builtin_bit_cast(uint32_t, p) << 32) | (0xffffffffu - (uint32_t)v);
      top = key > top ? key : top;
    }
    atomicMax(&best, top);
    __syncthreads();
    if (threadIdx.x == 0) a.next[b] = (int32_t)(0xffffffffu - (uint32_t)best);
    return;
  }
  const double want = u * total;
  int first = -1, last = -1;
  double at_first = 0.0, at_last = 0.0, base = 0.0;
  for (int i = c0; i < c1; ++i) {
    const double s = sums[i];
    if (s > 0.0) {
      last = i;
      at_last = run;
      if (run + s > want && first < 0) {
        first = i;
        at_first = run;
      }
    }
    run += s;
  }
  const int held = pick(pk, first, at_first, last, at_last, base);
  double r[8], t;
  const int v = held * kVerifyChunk + 8 * threadIdx.x;
  left8<PT>(a, e, row, v, r);
  run = chunk_scan(r, red, t);
  first = last = -1;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    run += r[i];
    if (r[i] > 0.0) {
      last = v + i;
      if (base + run > want && first < 0) first = v + i;
    }
  }
  const int next = pick(pk, first, 0.0, last, 0.0, base);
  if (threadIdx.x == 0) a.next[b] = next;
}

template <int PT>
void launch_p(const VerifyArgs& a, hipStream_t s) {
  if (a.draft)
    for (int k = 1; k < a.max_children; ++k)
      hipLaunchKernelGGL((verify_z_kernel<PT>), dim3(a.zblk, a.n_nodes), dim3(kVT), 0, s, a, k);
  hipLaunchKernelGGL((verify_sum_kernel<PT>), dim3(a.nblk, a.batch), dim3(kVT), 0, s, a);
  hipLaunchKernelGGL((verify_next_kernel<PT>), dim3(a.batch), dim3(kVT), 0, s, a);
}

}  // namespace

hipError_t launch_verify(const VerifyArgs& a, hipStream_t s) {
  switch (a.p_type) {
    case DWKV_F32: launch_p<DWKV_F32>(a, s); break;
    case DWKV_F16: launch_p<DWKV_F16>(a, s); break;
    default: launch_p<DWKV_BF16>(a, s); break;
  }
  return hipGetLastError();
}

}  // namespace dwkv
