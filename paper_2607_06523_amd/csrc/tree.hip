// The tree attention (tree_dev.h): the split pass for fp16 queries, the merge
// and the launches.
#include "tree_dev.h"

namespace dwkv {

void launch_tree_split_bf16(const TreeArgs& a, hipStream_t s);

namespace {

// Joins the partials of kMR rows and applies B^V.  The four waves take every
// fourth chunk with a running maximum and sum of their own, a lane four columns
// (residual channels, then a~): no load waits for another's value.  Sums in a
// fixed order.  Bound by latency: 5 us for 20 rows of 5 partials, 7.5 for 32 rows
// of 30 and for 256 of 5, 15 for 25 blocks of 32 rows in 16 sequences (traced); pairs
// of rows keep B^V's read (12 KB at r_b 48) below the partials' own.
// grid (row pairs of the longest sequence, Hkv, B)
constexpr int kMR = 2, kMW = 4;
struct alignas(16) MergeSmem {
  float part[kMW][kMR][2 * D];
  float m[kMW][kMR], l[kMW][kMR];
  float as[kMR][D];
};

__global__ __launch_bounds__(64 * kMW) void tree_merge_kernel(const TreeArgs a) {
  __shared__ MergeSmem sm;
  extern __shared__ u4v basis[];         // r_b rows of B^V
  const int b = blockIdx.z, h = blockIdx.y, H = a.n_kv_heads, rb = a.rb;
  const int wv = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const u4v* bv = reinterpret_cast<const u4v*>(a.basis + (int64_t)b * a.basis_b_stride + (int64_t)(h * 2 + 1) * rb * D);
  u4v bw[8];                             // B^V on its way to LDS
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i * 16 < rb) bw[i] = bv[threadIdx.x + 256 * i];
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
  const int stride = D + rb + 4, block = r0 / R;              // R is a multiple of kMR
  const float* p0 = a.part + ((base + block) * H + h) * R * stride + (int64_t)(r0 % R) * stride;
  const int64_t step = (int64_t)nrb * H * R * stride;    // to the next chunk's partial
  const float inf = __builtin_inff();
  const int cols = (D + rb) / 4, mycol = 4 * min(lane, cols - 1);
  f4 o[kMR] = {};
  float m[kMR], l[kMR];
#pragma unroll
  for (int r = 0; r < kMR; ++r) m[r] = -inf, l[r] = 0.f;
  constexpr int kAt = 4;                 // chunks of a wave read at once
  const int last_row = rows - 1 - r0;
  for (int s0 = wv; s0 <= chunks; s0 += kMW * kAt) {
    float2 ml[kAt][kMR];
    f4 x[kAt][kMR];
#pragma unroll
    for (int k = 0; k < kAt; ++k)
#pragma unroll
      for (int r = 0; r < kMR; ++r) {
        const float* p = p0 + min(r, last_row) * stride + min(s0 + kMW * k, chunks) * step;
        ml[k][r] = *reinterpret_cast<const float2*>(p + D + rb);
        x[k][r] = *reinterpret_cast<const f4*>(p + mycol);
      }
#pragma unroll
    for (int k = 0; k < kAt; ++k) {
      if (s0 + kMW * k > chunks) continue;
#pragma unroll
      for (int r = 0; r < kMR; ++r) {
        if (ml[k][r].y == 0.f) continue;   // nothing there
        const float mn = fmaxf(m[r], ml[k][r].x), was = m[r] > -inf ? __builtin_amdgcn_exp2f(m[r] - mn) : 0.f;
        const float wt = __builtin_amdgcn_exp2f(ml[k][r].x - mn);
        l[r] = ml[k][r].y < 0.f ? -inf : __builtin_fmaf(wt, ml[k][r].y, l[r] * was);   // absent: stays -inf
        o[r] = o[r] * was + x[k][r] * wt;
        m[r] = mn;
      }
    }
  }
  if (lane < cols) {
#pragma unroll
    for (int r = 0; r < kMR; ++r) *reinterpret_cast<f4*>(&sm.part[wv][r][4 * lane]) = o[r];
  }
  if (lane == 0) {
#pragma unroll
    for (int r = 0; r < kMR; ++r) sm.m[wv][r] = m[r], sm.l[wv][r] = l[r];
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i * 16 < rb) basis[threadIdx.x + 256 * i] = bw[i];
  __syncthreads();
  const int r = threadIdx.x >> 7, c = threadIdx.x & 127;     // a thread per output
  float ms = -inf, ls = 0.f, out = 0.f, av = 0.f;
  bool absent = false;
#pragma unroll
  for (int u = 0; u < kMW; ++u) ms = fmaxf(ms, sm.m[u][r]);
#pragma unroll
  for (int u = 0; u < kMW; ++u) {
    if (sm.l[u][r] == 0.f) continue;
    absent = absent || sm.l[u][r] == -inf;
    const float wt = __builtin_amdgcn_exp2f(sm.m[u][r] - ms);
    ls = __builtin_fmaf(wt, sm.l[u][r], ls);
    out = __builtin_fmaf(wt, sm.part[u][r][c], out);
    if (c < rb) av = __builtin_fmaf(wt, sm.part[u][r][D + c], av);
  }
  const float inv = ls == 0.f ? 0.f : 1.f / ls;
  out *= inv;
  sm.as[r][c] = c < rb ? av * inv : 0.f;
  __syncthreads();
  const uint16_t* bas = reinterpret_cast<const uint16_t*>(basis);
#pragma unroll 8
  for (int i = 0; i < rb; ++i) out = __builtin_fmaf(sm.as[r][i], half_bits_to_float(bas[i * D + c]), out);
  if (r0 + r < rows)
    a.out[((int64_t)(n0 + (r0 + r) / a.group) * a.n_q_heads + h * a.group + (r0 + r) % a.group) * D + c] = absent ? 0.f : out;
}

}  // namespace

hipError_t launch_tree(const TreeArgs& a, int max_rows, hipStream_t s) {
  if (a.q_bf16) launch_tree_split_bf16(a, s);
  else launch_tree_split<false>(a, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(tree_merge_kernel, dim3((max_rows + kMR - 1) / kMR, a.n_kv_heads, a.batch), dim3(64 * kMW), (unsigned)(a.rb * D * 2), s, a);
  return hipGetLastError();
}

}  // namespace dwkv
