// The tree attention (tree_dev.h): the split pass for fp16 queries, the merge
// and the launches.
#include "tree_dev.h"

namespace dwkv {

void launch_tree_split_bf16(const TreeArgs& a, hipStream_t s);

namespace {

// Joins the partials of kMR rows and applies B^V.  The four waves take every
// fourth chunk, a lane four columns (residual channels, then a~), so a row's
// partials are read with independent loads; sums in a fixed order.
// grid (row pairs of the longest sequence, Hkv, B)
constexpr int kMR = 2, kMW = 4;
struct alignas(16) MergeSmem {
  float part[kMW][kMR][2 * D];
  float m[kMW][kMR], l[kMW][kMR];
  float as[kMR][D];
  uint16_t basis[128 * D];
};

__global__ __launch_bounds__(64 * kMW) void tree_merge_kernel(const TreeArgs a) {
  __shared__ MergeSmem sm;
  const int b = blockIdx.z, h = blockIdx.y, H = a.n_kv_heads, rb = a.rb;
  const int wv = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int64_t base = 0;
  int t0, t1, n0, n;
  if (a.wt.n_seq > 0) {
    base = a.wt.work[b];
    t0 = a.wt.tok[b], t1 = a.wt.tok[b + 1], n0 = a.wt.node[b], n = a.wt.node[b + 1] - n0;
  } else {
    for (int i = lane; i < b; i += 64) {
      int ch, nr;
      seq_items(a.cu[i + 1] - a.cu[i], a.cu_nodes[i + 1] - a.cu_nodes[i], a, ch, nr);
      base += (int64_t)(ch + 1) * nr;
    }
    for (int d = 32; d; d >>= 1) base += __shfl_xor(base, d);
    t0 = a.cu[b], t1 = a.cu[b + 1], n0 = a.cu_nodes[b], n = a.cu_nodes[b + 1] - n0;
  }
  int chunks, nrb;
  seq_items(t1 - t0, n, a, chunks, nrb);
  const int r0 = blockIdx.x * kMR, rows = n * a.group;
  if (r0 >= rows) return;
  const uint16_t* bv = a.basis + (int64_t)b * a.basis_b_stride + (int64_t)(h * 2 + 1) * rb * D;
  for (int i = threadIdx.x; i < rb * (D / 8); i += 64 * kMW) reinterpret_cast<u4v*>(sm.basis)[i] = reinterpret_cast<const u4v*>(bv)[i];
  const int stride = D + rb + 4, block = r0 / a.rows;         // a.rows is a multiple of kMR
  const float* p0 = a.part + ((base + block) * H + h) * a.rows * stride + (int64_t)(r0 % a.rows) * stride;
  const int64_t step = (int64_t)nrb * H * a.rows * stride;    // to the next chunk's partial
  const float inf = __builtin_inff();
  // the rows' statistics: the largest reference, then every chunk's weight
  float ms[kMR], ls[kMR];
  bool absent[kMR];
#pragma unroll
  for (int r = 0; r < kMR; ++r) {
    ms[r] = -inf;
    bool gone = r0 + r >= rows;
    for (int s = lane; s <= chunks && r0 + r < rows; s += 64) {
      const float2 ml = *reinterpret_cast<const float2*>(p0 + r * stride + s * step + D + rb);
      gone = gone || ml.y < 0.f;
      if (!(ml.y == 0.f)) ms[r] = fmaxf(ms[r], ml.x);
    }
    for (int d = 32; d; d >>= 1) ms[r] = fmaxf(ms[r], __shfl_xor(ms[r], d));
    absent[r] = __ballot(gone) != 0;
    ls[r] = 0.f;
  }
  const int cols = (D + rb) / 4;
  f4 o[kMR][2] = {};
#pragma unroll
  for (int r = 0; r < kMR; ++r) {
    if (absent[r]) continue;
    const float* p = p0 + r * stride;
#pragma unroll 4
    for (int s = wv; s <= chunks; s += kMW) {
      const float2 ml = *reinterpret_cast<const float2*>(p + s * step + D + rb);
      const f4 x = *reinterpret_cast<const f4*>(p + s * step + 4 * min(lane, cols - 1));
      const float wt = ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - ms[r]);
      ls[r] = __builtin_fmaf(wt, ml.y, ls[r]);
      if (ml.y == 0.f) continue;         // nothing there, and its sums may be anything
      o[r][0] += x * wt;
    }
  }
  if (lane < cols) {
#pragma unroll
    for (int r = 0; r < kMR; ++r) *reinterpret_cast<f4*>(&sm.part[wv][r][4 * lane]) = o[r][0];
  }
  if (lane == 0) {
#pragma unroll
    for (int r = 0; r < kMR; ++r) sm.l[wv][r] = ls[r];
  }
  __syncthreads();
  const int r = threadIdx.x >> 7, c = threadIdx.x & 127;     // a thread per output
  float l = 0.f, out = 0.f, av = 0.f;
#pragma unroll
  for (int u = 0; u < kMW; ++u) {
    l += sm.l[u][r];
    out += sm.part[u][r][c];
    if (c < rb) av += sm.part[u][r][D + c];
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  out *= inv;
  sm.as[r][c] = c < rb ? av * inv : 0.f;
  __syncthreads();
#pragma unroll 8
  for (int i = 0; i < rb; ++i) out = __builtin_fmaf(sm.as[r][i], half_bits_to_float(sm.basis[i * D + c]), out);
  if (r0 + r < rows)
    a.out[((int64_t)(n0 + (r0 + r) / a.group) * a.n_q_heads + h * a.group + (r0 + r) % a.group) * D + c] = absent[r] ? 0.f : out;
}

}  // namespace

hipError_t launch_tree(const TreeArgs& a, int max_rows, hipStream_t s) {
  if (a.q_bf16) launch_tree_split_bf16(a, s);
  else launch_tree_split<false>(a, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(tree_merge_kernel, dim3((max_rows + kMR - 1) / kMR, a.n_kv_heads, a.batch), dim3(64 * kMW), 0, s, a);
  return hipGetLastError();
}

}  // namespace dwkv
