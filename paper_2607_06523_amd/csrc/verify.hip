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
// Bound by latency: a call reads few rows.  Sums are float64 in a fixed order
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

// A sequence's nodes, one per lane: parent row (inside the sequence), place
// among its parent's children, and the numbers of its test.
struct Node {
  int parent, place;
  double u, p, q;
};

template <int PT>
__device__ __forceinline__ Node load_node(const VerifyArgs& a, int n0, int n, int lane, int* lds) {
  Node d;
  d.parent = -1;
  d.u = d.p = d.q = 0.0;
  if (lane > 0 && lane < n) {
    const int p = a.parent[n0 + lane];
    if (p >= 0 && p < lane) d.parent = p;
    const int x = a.token[n0 + lane];
    d.u = (double)a.u[n0 + lane];
    if (d.parent >= 0 && x >= 0 && x < a.vocab) {
      d.p = prob<PT>(a.target, (int64_t)(n0 + d.parent) * a.vocab + x);
      if (a.draft) d.q = prob<PT>(a.draft, (int64_t)(n0 + d.parent) * a.vocab + x);
    }
  }
  lds[lane] = d.parent;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  d.place = 0;
  for (int j = 1; j < lane; ++j) d.place += lds[j] == d.parent;
  if (d.parent < 0 || d.place >= a.max_children) d.parent = -1;
  return d;
}

// Z_k of row `row` (k >= 1), the chunks' sums in order.
__device__ __forceinline__ double row_z(const VerifyArgs& a, int row, int k) {
  const double* z = a.z + ((int64_t)row * (a.max_children - 1) + (k - 1)) * a.zblk;
  double s = 0.0;
  for (int i = 0; i < a.zblk; ++i) s += z[i];
  return s;
}

// Tests the children of node `at` in order; the one that stands, or -1.  At
// most `limit` rejections are looked at; k counts them, c is theirs.
__device__ __forceinline__ int test_children(const VerifyArgs& a, int n0, const Node& d, const int* token, int at, int limit,
                                             int lane, int& k, double& c, unsigned long long& out) {
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
      if (kids && k < limit) Z = row_z(a, n0 + at, k);
    } else {
      bool again = false;                // a token rejected before is left out already
      for (unsigned long long o = out; o; o &= o - 1) again |= token[__ffsll(o) - 1] == token[j];
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
  __shared__ int lds[MN], tok[MN];
  __shared__ double red[kVT / 64], sc;
  __shared__ int need;
  const int row = blockIdx.y, lane = threadIdx.x & 63;
  if (threadIdx.x < 64) {
    int b = 0, hi = a.batch;             // the row's sequence: cu[b] <= row < cu[hi]
    while (hi - b > 1) {
      const int mid = (b + hi) >> 1;
      if (a.cu_nodes[mid] <= row) b = mid; else hi = mid;
    }
    while (a.cu_nodes[b + 1] <= row) ++b;
    const int n0 = a.cu_nodes[b], n = a.cu_nodes[b + 1] - n0;
    const Node d = load_node<PT>(a, n0, n, lane, lds);
    tok[lane] = 0;
    int tried;
    double c = 0.0;
    unsigned long long out;
    const int kids = __popcll(__ballot(d.parent == row - n0));
    int stands = -1;
    if (kids > k) stands = test_children(a, n0, d, tok, row - n0, k, lane, tried, c, out);
    if (lane == 0) {
      need = kids > k && stands < 0;
      sc = c;
    }
  }
  __syncthreads();
  if (!need) return;
  const int v0 = blockIdx.x * kVerifyZChunk, v1 = min(v0 + kVerifyZChunk, a.vocab);
  const int64_t at = (int64_t)row * a.vocab;
  double s = 0.0;
  for (int v = v0 + threadIdx.x; v < v1; v += kVT) s += fmax(prob<PT>(a.target, at + v) - sc * prob<PT>(a.draft, at + v), 0.0);
  s = block_sum(s, red);
  if (threadIdx.x == 0) a.z[((int64_t)row * (a.max_children - 1) + (k - 1)) * a.zblk + blockIdx.x] = s;
}

// r of entries v .. v + 7 of the last row, past the end 0.
template <int PT>
__device__ __forceinline__ void left8(const VerifyArgs& a, const VerifyEnd& e, int64_t row, int v, double (&r)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    r[i] = 0.0;
    if (v + i < a.vocab) {
      r[i] = prob<PT>(a.target, row * a.vocab + v + i);
      if (e.c > 0.0) r[i] = fmax(r[i] - e.c * prob<PT>(a.draft, row * a.vocab + v + i), 0.0);
    }
  }
  for (int j = 0; j < e.n_out; ++j) {
    const int x = e.out[j] - v;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (x == i) r[i] = 0.0;
  }
}

// Running sum before this thread's eight entries, and the chunk's sum: the same
// additions in both kernels.
__device__ __forceinline__ double chunk_scan(const double (&r)[8], double* red, double& total) {
  double mine = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) mine += r[i];
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

// grid (nblk, B)
template <int PT>
__global__ __launch_bounds__(kVT) void verify_sum_kernel(const VerifyArgs a) {
  __shared__ int lds[MN], tok[MN];
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
    const Node d = load_node<PT>(a, n0, n, lane, lds);
    tok[lane] = lane < n ? a.token[n0 + lane] : 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    int at = 0, kept = 1, k;
    int path = lane == 0 ? 0 : -1;
    double c;
    unsigned long long out;
    for (;;) {
      const int j = test_children(a, n0, d, tok, at, a.max_children, lane, k, c, out);
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
    if ((out >> lane) & 1) e.out[__popcll(out & ((1ull << lane) - 1))] = tok[lane];
    if (writes) {
      if (lane < n) a.path[n0 + lane] = path;
      if (lane == 0) a.n_kept[b] = kept;
    }
  }
  __syncthreads();
  if (writes && threadIdx.x == 0) a.end[b] = e;
  double r[8], total;
  left8<PT>(a, e, n0 + e.node, blockIdx.x * kVerifyChunk + 8 * threadIdx.x, r);
  chunk_scan(r, red, total);
  if (threadIdx.x == 0) a.sum[(int64_t)b * a.nblk + blockIdx.x] = total;
}

// grid (B)
template <int PT>
__global__ __launch_bounds__(kVT) void verify_next_kernel(const VerifyArgs a) {
  __shared__ double red[kVT / 64];
  __shared__ VerifyEnd e;
  __shared__ double base, total;
  __shared__ int chunk, found;
  __shared__ unsigned long long best;
  const int b = blockIdx.x;
  if (threadIdx.x == 0) {
    e = a.end[b];
    found = 0x7fffffff;
    best = 0;
    if (e.node >= 0) {                   // the chunks' sums in order
      const double* s = a.sum + (int64_t)b * a.nblk;
      double t = 0.0;
      for (int i = 0; i < a.nblk; ++i) t += s[i];
      total = t;
      const double want = (double)a.u_next[b] * t;
      double run = 0.0;
      base = 0.0;
      chunk = -1;
      for (int i = 0; i < a.nblk; ++i) {
        if (s[i] > 0.0) {                // the last chunk with something left, should rounding pass them all
          base = run;
          chunk = i;
        }
        run += s[i];
        if (run > want) break;
      }
    }
  }
  __syncthreads();
  if (e.node < 0) {
    if (threadIdx.x == 0) a.next[b] = -1;
    return;
  }
  const int64_t row = a.cu_nodes[b] + e.node;
  if (!(total > 0.0)) {                  // nothing left: the first largest p
    unsigned long long mine = 0;
    for (int v = threadIdx.x; v < a.vocab; v += kVT) {
      const float p = (float)prob<PT>(a.target, row * a.vocab + v);
      const unsigned long long key = ((unsigned long long)__builtin_bit_cast(uint32_t, p) << 32) | (0xffffffffu - (uint32_t)v);
      mine = key > mine ? key : mine;
    }
    atomicMax(&best, mine);
    __syncthreads();
    if (threadIdx.x == 0) a.next[b] = (int32_t)(0xffffffffu - (uint32_t)best);
    return;
  }
  double r[8], t;
  const int v = chunk * kVerifyChunk + 8 * threadIdx.x;
  left8<PT>(a, e, row, v, r);
  double run = chunk_scan(r, red, t);
  const double want = (double)a.u_next[b] * total;
  int hit = 0x7fffffff, last = -1;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    run += r[i];
    if (r[i] > 0.0) {
      last = v + i;
      if (base + run > want && hit == 0x7fffffff) hit = v + i;
    }
  }
  atomicMin(&found, hit);
  atomicMax(&best, (unsigned long long)(last + 1));
  __syncthreads();
  if (threadIdx.x == 0) a.next[b] = found != 0x7fffffff ? found : (int32_t)best - 1;
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
