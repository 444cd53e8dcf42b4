// Repacking of a factorized cache: copies, forks, compacts, frees and grows
// sequences (gfx950).  Nothing is computed but the offsets; every byte of the
// destination is written once, from where its token lay in the source:
//  * repack_code_kernel: the tokens' rank codes, and the block sums of their ranks
//  * repack_offset_kernel: the offsets, each block adding the sums before it
//  * repack_copy_kernel: coefficients, scales and entries of 64 tokens of one
//    (layer, Z, KV head) per workgroup.
#include "entry.h"
#include "internal.h"

namespace dwkv {
namespace {

typedef uint32_t u4v __attribute__((ext_vector_type(4)));

constexpr int kRT = 256;
constexpr int kTok = 64;                 // tokens per copy workgroup
constexpr int D = kHeadDim;

// Source token of slot t, or -1 for a fresh slot.
__device__ __forceinline__ int source(const RepackArgs& a, int64_t t) {
  const int s = a.src_token[t];
  return s >= 0 && s < a.T0 ? s : -1;
}

__device__ __forceinline__ int code_of(const RepackArgs& a, int mh, int64_t t) {
  const int s = a.src_token[t];
  int c = 0;
  if (s >= 0) {
    if (s < a.T0) c = a.from.rank_code[(int64_t)mh * a.T0 + s];
  } else if (a.new_code && -1 - (int64_t)s < a.n_new) {
    c = a.new_code[(int64_t)mh * a.n_new + (-1 - (int64_t)s)];
  }
  return c < a.n_levels ? c : 0;
}

__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* red, uint32_t& total) {   // exclusive
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  uint32_t inc = v;
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(inc, d);
    if (lane >= d) inc += o;
  }
  __syncthreads();
  if (lane == 63) red[wv] = inc;
  __syncthreads();
  uint32_t before = 0;
  total = 0;
  for (int i = 0; i < kRT / 64; ++i) {
    if (i < wv) before += red[i];
    total += red[i];
  }
  return before + inc - v;
}

// grid (nblk, M*Hkv)
__global__ __launch_bounds__(kRT) void repack_code_kernel(const RepackArgs a) {
  __shared__ uint32_t red[kRT / 64];
  const int mh = blockIdx.y;
  uint8_t* code = const_cast<uint8_t*>(a.to.rank_code) + (int64_t)mh * a.T;
  uint32_t sum = 0;
  for (int i = 0; i < kRepackBlock / kRT; ++i) {
    const int64_t t = (int64_t)blockIdx.x * kRepackBlock + i * kRT + threadIdx.x;
    if (t < a.T) {
      const int c = code_of(a, mh, t);
      code[t] = (uint8_t)c;
      sum += (uint32_t)a.levels[c];
    }
  }
  uint32_t total;
  block_scan(sum, red, total);
  if (threadIdx.x == 0) a.bsum[(int64_t)mh * a.nblk + blockIdx.x] = total;
}

// grid (nblk, M*Hkv); also the bases, spread over the workgroups
__global__ __launch_bounds__(kRT) void repack_offset_kernel(const RepackArgs a) {
  __shared__ uint32_t red[kRT / 64];
  const int mh = blockIdx.y;
  const uint8_t* code = a.to.rank_code + (int64_t)mh * a.T;
  uint32_t* off = const_cast<uint32_t*>(a.to.res_off) + (int64_t)mh * (a.T + 1);
  uint32_t run = 0;
  {
    uint32_t sum = 0, total;
    for (int i = threadIdx.x; i < (int)blockIdx.x; i += kRT) sum += a.bsum[(int64_t)mh * a.nblk + i];
    block_scan(sum, red, total);
    run = total;
  }
  for (int i = 0; i < kRepackBlock / kRT; ++i) {
    const int64_t t = (int64_t)blockIdx.x * kRepackBlock + i * kRT + threadIdx.x;
    const uint32_t r = t < a.T ? (uint32_t)a.levels[code[t]] : 0u;
    uint32_t total;
    const uint32_t at = run + block_scan(r, red, total);
    if (t < a.T) {
      off[t] = at;
      if (t == a.T - 1) off[a.T] = at + r;
    }
    run += total;
  }
  if (a.T == 0 && threadIdx.x == 0 && blockIdx.x == 0) off[0] = 0;
  // bases of this window and head, both Z
  const int M = a.n_layers / a.window, n16 = 2 * a.rb * D / 8;
  for (int b = blockIdx.x; b < a.batch; b += gridDim.x) {
    const int sb = a.src_seq[b];
    if (sb < 0 || sb >= a.batch0) continue;
    const int64_t mhs = (int64_t)M * a.n_kv_heads;
    const u4v* s = static_cast<const u4v*>(a.from.basis) + ((int64_t)sb * mhs + mh) * n16;
    u4v* d = static_cast<u4v*>(const_cast<void*>(a.to.basis)) + ((int64_t)b * mhs + mh) * n16;
    for (int i = threadIdx.x; i < n16; i += kRT) d[i] = s[i];
  }
}

// grid (ceil(T16 / 64), Hkv, 2 L)
__global__ __launch_bounds__(kRT) void repack_copy_kernel(const RepackArgs a) {
  __shared__ int src[kTok];
  const int h = blockIdx.y, l = blockIdx.z >> 1, z = blockIdx.z & 1, H = a.n_kv_heads, rb = a.rb;
  const int64_t t0 = (int64_t)blockIdx.x * kTok, T16 = (a.T + 15) / 16 * 16, T160 = (a.T0 + 15) / 16 * 16;
  const int nt = (int)min((int64_t)kTok, T16 - t0), nr = (int)min((int64_t)kTok, a.T - t0);
  if (threadIdx.x < kTok) src[threadIdx.x] = (int)threadIdx.x < nr ? source(a, t0 + threadIdx.x) : -1;
  __syncthreads();
  const int64_t slab = (int64_t)l * H + h, zslab = ((int64_t)l * 2 + z) * H + h;
  const int esz = a.c8 ? 1 : 2;
  const uint8_t* cs = static_cast<const uint8_t*>(z ? a.from.coef_v : a.from.coef_k) + slab * T160 * rb * esz;
  uint8_t* cd = static_cast<uint8_t*>(const_cast<void*>(z ? a.to.coef_v : a.to.coef_k)) + slab * T16 * rb * esz;
  if (z == 0) {                          // key tiles: 16 bytes of one token
    const int per = rb * esz / 16;
    for (int i = threadIdx.x; i < nt * per; i += kRT) {
      const int tile = i / (16 * per), piece = i / 16 % per, k = tile * 16 + (i & 15), s = src[k];
      u4v w = {0, 0, 0, 0};
      if (s >= 0) w = *reinterpret_cast<const u4v*>(cs + (((int64_t)(s >> 4) * per + piece) * 16 + (s & 15)) * 16);
      *reinterpret_cast<u4v*>(cd + (((t0 >> 4) + tile) * per + piece) * 256 + (i & 15) * 16) = w;
    }
  } else {                               // value blocks: 16 bytes of one coefficient, 8 or 16 tokens
    const int tb = 16 / esz;
    for (int i = threadIdx.x; i < nt / tb * rb; i += kRT) {
      const int blk = i / rb, c = i % rb;
      u4v w = {0, 0, 0, 0};
      for (int j = 0; j < tb; ++j) {
        const int s = src[blk * tb + j];
        if (s < 0) continue;
        const uint8_t* p = cs + ((int64_t)(s / tb) * rb + c) * 16 + (s % tb) * esz;
        const uint32_t v = a.c8 ? *p : *reinterpret_cast<const uint16_t*>(p);
        w[j * esz / 4] |= v << (8 * (j * esz % 4));
      }
      *reinterpret_cast<u4v*>(cd + ((t0 / tb + blk) * rb + c) * 16) = w;
    }
  }
  const uint16_t* ss = static_cast<const uint16_t*>(a.from.res_scale) + zslab * a.T0;
  uint16_t* sd = static_cast<uint16_t*>(const_cast<void*>(a.to.res_scale)) + zslab * a.T;
  if ((int)threadIdx.x < nr) sd[t0 + threadIdx.x] = src[threadIdx.x] >= 0 ? ss[src[threadIdx.x]] : 0;
  if (a.c8) {
    const int nb = rb / 16;
    const uint16_t* bs = static_cast<const uint16_t*>(z ? a.from.coef_v_scale : a.from.coef_k_scale) + slab * nb * a.T0;
    uint16_t* bd = static_cast<uint16_t*>(const_cast<void*>(z ? a.to.coef_v_scale : a.to.coef_k_scale)) + slab * nb * a.T;
    for (int i = threadIdx.x; i < nb * kTok; i += kRT) {
      const int k = i % kTok, s = i / kTok;
      if (k < nr) bd[s * a.T + t0 + k] = src[k] >= 0 ? bs[s * a.T0 + src[k]] : 0;
    }
  }
  // entries: four lanes per token, two entries (one code byte) each in turn
  const int mh = (l / a.window) * H + h;
  const uint32_t* off = a.to.res_off + (int64_t)mh * (a.T + 1);
  const uint32_t* off0 = a.from.res_off + (int64_t)mh * (a.T0 + 1);
  const uint8_t* is = a.from.res_idx + zslab * a.stride0;
  const uint8_t* vs = a.from.res_val + zslab * (a.stride0 / 2);
  uint8_t* id = const_cast<uint8_t*>(a.to.res_idx) + zslab * a.stride;
  uint8_t* vd = const_cast<uint8_t*>(a.to.res_val) + zslab * (a.stride / 2);
  const int k = threadIdx.x >> 2;
  if (k < nr) {
    const uint32_t d0 = off[t0 + k], n = off[t0 + k + 1] - d0;
    const int s = src[k];
    const uint32_t s0 = s >= 0 ? off0[s] : 0;
    for (uint32_t e = 2 * (threadIdx.x & 3); e < n; e += 8) {
      if ((int64_t)d0 + e + 2 > a.stride - kResTailPad) break;
      uint16_t ch = (uint16_t)(e | (e + 1) << 8);
      uint8_t v = 0;
      if (s >= 0) {
        if ((int64_t)s0 + e + 2 > a.stride0) break;
        ch = *reinterpret_cast<const uint16_t*>(is + s0 + e);
        v = vs[(s0 + e) >> 1];
      }
      *reinterpret_cast<uint16_t*>(id + d0 + e) = ch;
      vd[(d0 + e) >> 1] = v;
    }
  }
}

}  // namespace

hipError_t launch_repack(const RepackArgs& a, hipStream_t s) {
  const dim3 scan(a.nblk, a.n_layers / a.window * a.n_kv_heads);
  hipLaunchKernelGGL(repack_code_kernel, scan, dim3(kRT), 0, s, a);
  hipLaunchKernelGGL(repack_offset_kernel, scan, dim3(kRT), 0, s, a);
  const unsigned tiles = (unsigned)((a.T + kTok - 1) / kTok);
  if (tiles > 0) hipLaunchKernelGGL(repack_copy_kernel, dim3(tiles, a.n_kv_heads, 2 * a.n_layers), dim3(kRT), 0, s, a);
  return hipGetLastError();
}

}  // namespace dwkv
