// Repacking of a factorized cache: copies, forks, compacts, frees and grows
// sequences (gfx950).  Nothing is computed but the offsets; every byte of the
// destination is written once, from where its token lay in the source:
//  * repack_code_kernel: the tokens' rank codes, and the block sums of their ranks
//  * repack_offset_kernel: the offsets, each block adding the sums before it (a
//    cache of one block has them from the first kernel)
//  * repack_copy_kernel: coefficients, scales and entries of 256 tokens of one
//    (layer, KV head) per workgroup, keys and values.
// Bound by HBM, reading and writing: a cache of 65536 tokens (4 layers, 8 KV heads, r_b
// 48) that grows by 64 slots moves 853 MB in 177 us, 4.8 TB/s, as fast as a plain
// copy of 2 GiB on the device.  256 tokens per workgroup: whole 16-byte pieces of keys
// and values go from source to destination without LDS, and a value block whose tokens
// follow each other in the source is two reads and a shift.
#include "entry.h"
#include "internal.h"

namespace dwkv {
namespace {

typedef uint32_t u4v __attribute__((ext_vector_type(4)));

constexpr int kRT = 256;
constexpr int kTok = kRT;                // tokens per copy workgroup, one per thread
constexpr int kPer = kRepackBlock / kRT; // tokens per thread of the offset scan
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

// Offsets of a block whose tokens' ranks come after `run` entries, four
// consecutive tokens per thread; the block's total.
__device__ __forceinline__ uint32_t write_offsets(const RepackArgs& a, int mh, const int (&code)[kPer], uint32_t run, uint32_t* red) {
  uint32_t* off = const_cast<uint32_t*>(a.to.res_off) + (int64_t)mh * (a.T + 1);
  const int64_t t0 = (int64_t)blockIdx.x * kRepackBlock + kPer * threadIdx.x;
  uint32_t mine = 0, total;
#pragma unroll
  for (int i = 0; i < kPer; ++i) mine += t0 + i < a.T ? (uint32_t)a.levels[code[i]] : 0u;
  uint32_t at = run + block_scan(mine, red, total);
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (t0 + i >= a.T) break;
    off[t0 + i] = at;
    at += (uint32_t)a.levels[code[i]];
    if (t0 + i == a.T - 1) off[a.T] = at;
  }
  if (a.T == 0 && blockIdx.x == 0 && threadIdx.x == 0) off[0] = 0;
  return total;
}

// Bases of a window and head, both Z, spread over the blocks.
__device__ __forceinline__ void copy_bases(const RepackArgs& a, int mh) {
  const int M = a.n_layers / a.window, n16 = 2 * a.rb * D / 8;
  for (int b = blockIdx.x; b < a.batch; b += gridDim.x) {
    const int sb = a.src_seq[b];
    if (sb < 0 || sb >= a.batch0) continue;
    const int64_t mhs = (int64_t)M * a.n_kv_heads;
    const u4v* s = static_cast<const u4v*>(a.from.basis) + ((int64_t)sb * mhs + mh) * n16;
    u4v* d = static_cast<u4v*>(const_cast<void*>(a.to.basis)) + ((int64_t)b * mhs + mh) * n16;
#pragma unroll 4
    for (int i = threadIdx.x; i < n16; i += kRT) d[i] = s[i];
  }
}

// grid (nblk, M*Hkv)
__global__ __launch_bounds__(kRT) void repack_code_kernel(const RepackArgs a) {
  __shared__ uint32_t red[kRT / 64];
  const int mh = blockIdx.y;
  uint8_t* to = const_cast<uint8_t*>(a.to.rank_code) + (int64_t)mh * a.T;
  const int64_t t0 = (int64_t)blockIdx.x * kRepackBlock + kPer * threadIdx.x;
  int code[kPer];
  uint32_t sum = 0, total;
#pragma unroll
  for (int i = 0; i < kPer; ++i) code[i] = t0 + i < a.T ? code_of(a, mh, t0 + i) : 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (t0 + i < a.T) {
      to[t0 + i] = (uint8_t)code[i];
      sum += (uint32_t)a.levels[code[i]];
    }
  if (a.nblk == 1) {
    write_offsets(a, mh, code, 0, red);
    copy_bases(a, mh);
    return;
  }
  block_scan(sum, red, total);
  if (threadIdx.x == 0) a.bsum[(int64_t)mh * a.nblk + blockIdx.x] = total;
}

// grid (nblk, M*Hkv)
__global__ __launch_bounds__(kRT) void repack_offset_kernel(const RepackArgs a) {
  __shared__ uint32_t red[kRT / 64];
  const int mh = blockIdx.y;
  const uint8_t* from = a.to.rank_code + (int64_t)mh * a.T;
  const int64_t t0 = (int64_t)blockIdx.x * kRepackBlock + kPer * threadIdx.x;
  int code[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) code[i] = t0 + i < a.T ? from[t0 + i] : 0;
  uint32_t sum = 0, before;
  for (int i = threadIdx.x; i < (int)blockIdx.x; i += kRT) sum += a.bsum[(int64_t)mh * a.nblk + i];
  block_scan(sum, red, before);
  write_offsets(a, mh, code, before, red);
  copy_bases(a, mh);
}

// 16 bytes from byte `sh` (0 .. 15) of the 32 bytes lo, hi.
__device__ __forceinline__ u4v funnel(u4v lo, u4v hi, int sh) {
  typedef unsigned long long u64;
  const u64 w0 = lo.x | (u64)lo.y << 32, w1 = lo.z | (u64)lo.w << 32, w2 = hi.x | (u64)hi.y << 32, w3 = hi.z | (u64)hi.w << 32;
  const u64 a0 = sh & 8 ? w1 : w0, a1 = sh & 8 ? w2 : w1, a2 = sh & 8 ? w3 : w2;
  const int r = 8 * (sh & 7);
  const u64 o0 = r ? a0 >> r | a1 << (64 - r) : a0, o1 = r ? a1 >> r | a2 << (64 - r) : a1;
  return u4v{(uint32_t)o0, (uint32_t)(o0 >> 32), (uint32_t)o1, (uint32_t)(o1 >> 32)};
}

// grid (ceil(T16 / 256), Hkv, L)
template <bool C8>
__global__ __launch_bounds__(kRT) void repack_copy_kernel(const RepackArgs a) {
  constexpr int esz = C8 ? 1 : 2, tb = 16 / esz;       // bytes of a coefficient; tokens of a value block
  __shared__ int src[kTok], run[kTok / tb];            // run: first source token of a block of consecutive ones, else -1
  __shared__ uint32_t off[kTok + 1], from[kTok];       // first entries here and there
  const int h = blockIdx.y, l = blockIdx.z, H = a.n_kv_heads, rb = a.rb, tid = threadIdx.x;
  const int64_t t0 = (int64_t)blockIdx.x * kTok, T16 = (a.T + 15) / 16 * 16, T160 = (a.T0 + 15) / 16 * 16;
  const int nt = (int)min((int64_t)kTok, T16 - t0), nr = (int)min((int64_t)kTok, a.T - t0);
  const int mh = (l / a.window) * H + h;
  const uint32_t* off_to = a.to.res_off + (int64_t)mh * (a.T + 1) + t0;
  const int s = tid < nr ? source(a, t0 + tid) : -1;
  const uint32_t o = off_to[min(tid, nr)];
  if (tid == 0) off[kTok] = off_to[nr];
  src[tid] = s;
  off[tid] = o;
  from[tid] = s >= 0 ? a.from.res_off[(int64_t)mh * (a.T0 + 1) + s] : 0u;
  {
    int ok = s >= 0;                     // consecutive tokens of a value block, looked for with lane shifts
    const int first = __shfl(s, (tid & 63) & ~(tb - 1));
    ok = ok && s == first + (tid & (tb - 1));
    const unsigned long long all = __ballot(ok);
    if ((tid & (tb - 1)) == 0) run[tid / tb] = ((all >> (tid & 63)) & ((1ull << tb) - 1)) == (1ull << tb) - 1 ? s : -1;
  }
  __syncthreads();
  const int64_t slab = (int64_t)l * H + h;
  // ---- key tiles: a thread's token, 16 bytes at a time
  {
    const int per = rb * esz / 16;
    const uint8_t* cs = static_cast<const uint8_t*>(a.from.coef_k) + slab * T160 * rb * esz + ((int64_t)(max(s, 0) >> 4) * per * 16 + (max(s, 0) & 15)) * 16;
    uint8_t* cd = static_cast<uint8_t*>(const_cast<void*>(a.to.coef_k)) + slab * T16 * rb * esz + (((t0 + tid) >> 4) * per * 16 + (tid & 15)) * 16;
    if (tid < nt) {
#pragma unroll 8
      for (int p = 0; p < per; ++p) {
        u4v w = {0, 0, 0, 0};
        if (s >= 0) w = *reinterpret_cast<const u4v*>(cs + p * 256);
        *reinterpret_cast<u4v*>(cd + p * 256) = w;
      }
    }
  }
  // ---- value blocks: 16 bytes of one coefficient, the block's tokens
  {
    const uint8_t* cs = static_cast<const uint8_t*>(a.from.coef_v) + slab * T160 * rb * esz;
    uint8_t* cd = static_cast<uint8_t*>(const_cast<void*>(a.to.coef_v)) + slab * T16 * rb * esz + t0 * rb * esz;
    const int n = nt / tb * rb;
    int blk = tid / rb, c = tid % rb;
    const int dblk = kRT / rb, dc = kRT % rb;
#pragma unroll 4
    for (int i = tid; i < n; i += kRT) {
      const int s0 = run[blk];
      u4v w = {0, 0, 0, 0};
      if (s0 >= 0) {
        const int sh = s0 % tb * esz;
        const uint8_t* p = cs + ((int64_t)(s0 / tb) * rb + c) * 16;
        w = *reinterpret_cast<const u4v*>(p);
        if (sh) w = funnel(w, *reinterpret_cast<const u4v*>(p + rb * 16), sh);
      } else {
        for (int j = 0; j < tb; ++j) {
          const int t = src[blk * tb + j];
          if (t < 0) continue;
          const uint8_t* p = cs + ((int64_t)(t / tb) * rb + c) * 16 + (t % tb) * esz;
          const uint32_t v = C8 ? *p : *reinterpret_cast<const uint16_t*>(p);
          w[j * esz / 4] |= v << (8 * (j * esz % 4));
        }
      }
      *reinterpret_cast<u4v*>(cd + (int64_t)i * 16) = w;
      c += dc;
      blk += dblk;
      if (c >= rb) c -= rb, ++blk;
    }
  }
  // ---- scales
  if (tid < nr) {
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const int64_t zslab = ((int64_t)l * 2 + z) * H + h;
      const uint16_t* ss = static_cast<const uint16_t*>(a.from.res_scale) + zslab * a.T0;
      uint16_t* sd = static_cast<uint16_t*>(const_cast<void*>(a.to.res_scale)) + zslab * a.T;
      sd[t0 + tid] = s >= 0 ? ss[s] : 0;
      if constexpr (C8) {
        const int nb = rb / 16;
        const uint16_t* bs = static_cast<const uint16_t*>(z ? a.from.coef_v_scale : a.from.coef_k_scale) + slab * nb * a.T0;
        uint16_t* bd = static_cast<uint16_t*>(const_cast<void*>(z ? a.to.coef_v_scale : a.to.coef_k_scale)) + slab * nb * a.T;
#pragma unroll 4
        for (int k = 0; k < nb; ++k) bd[k * a.T + t0 + tid] = s >= 0 ? bs[k * a.T0 + s] : 0;
      }
    }
  }
  // ---- entries, a pair of one token (ranks are even) per thread: two channel
  // bytes and one code byte, keys and values at the same place
  const int64_t zs = H * a.stride, zs0 = H * a.stride0;       // from keys to values
  const uint8_t* is = a.from.res_idx + ((int64_t)l * 2 * H + h) * a.stride0;
  const uint8_t* vs = a.from.res_val + ((int64_t)l * 2 * H + h) * (a.stride0 / 2);
  uint8_t* id = const_cast<uint8_t*>(a.to.res_idx) + ((int64_t)l * 2 * H + h) * a.stride;
  uint8_t* vd = const_cast<uint8_t*>(a.to.res_val) + ((int64_t)l * 2 * H + h) * (a.stride / 2);
  const uint32_t e0 = off[0];
  const int64_t room = min((int64_t)off[kTok], a.stride - kResTailPad) - e0;
  for (int64_t x = 2 * tid; x + 2 <= room; x += 2 * kRT) {
    const uint32_t e = e0 + (uint32_t)x;
    int k = 0;                           // the last token with off[k] <= e
#pragma unroll
    for (int d = kTok / 2; d; d >>= 1)
      if (off[k + d] <= e) k += d;
    const uint32_t j = e - off[k];
    uint16_t ch[2];
    uint8_t v[2] = {0, 0};
    ch[0] = ch[1] = (uint16_t)(j | (j + 1) << 8);
    if (src[k] >= 0) {
      const int64_t f = (int64_t)from[k] + j;
      if (f + 2 > a.stride0) continue;   // past the source's slab: its offsets are not its own
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        ch[z] = *reinterpret_cast<const uint16_t*>(is + z * zs0 + f);
        v[z] = vs[z * (zs0 / 2) + (f >> 1)];
      }
    }
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      *reinterpret_cast<uint16_t*>(id + z * zs + e) = ch[z];
      vd[z * (zs / 2) + (e >> 1)] = v[z];
    }
  }
}

}  // namespace

hipError_t launch_repack(const RepackArgs& a, hipStream_t s) {
  const dim3 scan(a.nblk, a.n_layers / a.window * a.n_kv_heads);
  hipLaunchKernelGGL(repack_code_kernel, scan, dim3(kRT), 0, s, a);
  if (a.nblk > 1) hipLaunchKernelGGL(repack_offset_kernel, scan, dim3(kRT), 0, s, a);
  const unsigned tiles = (unsigned)((a.T + kTok - 1) / kTok);
  const dim3 grid(tiles, a.n_kv_heads, a.n_layers);
  if (tiles > 0) {
    if (a.c8) hipLaunchKernelGGL(repack_copy_kernel<true>, grid, dim3(kRT), 0, s, a);
    else hipLaunchKernelGGL(repack_copy_kernel<false>, grid, dim3(kRT), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace dwkv
