// Attention of a tree of drafted tokens over the cross-depth factorized KV
// cache (Eq. 1 used through its linearity, as in the decode), gfx950.
//
// Row r of a sequence and KV head is node r / G, group member r % G.  For
// cached token t, with q~ = B^K q (once per workgroup, float32 MFMA):
//   S[t][r] = A^K_t . q~_r + s^K_t (R^K_t . q_r),   p = 2^(S - m_r)
//   O_r = (sum_t p A^V_t) B^V + sum_t (p s^V_t) R^V_t,  then the drafted nodes
// A decode has G rows; here G n of them share every byte read, so both sums
// and the routed residuals run on the matrix cores: a wave turns the entries
// of 32 tokens into dense code tiles in LDS (integers, exact in 16 bits) and
// multiplies them like the coefficients.
//
//  * tree_split_kernel: workgroup = (chunk of a sequence's tokens, KV head,
//    block of 16 NC rows), 8 waves taking its 32-token tiles in turn.  Scores
//    come out transposed, tokens down the accumulator and rows across, which is
//    the operand layout the value products read: probabilities never leave the
//    registers.  A tile's tokens are dealt to the score rows so that a lane's
//    eight scores are eight consecutive tokens, one value block.
//  * one more workgroup per (sequence, KV head, row block) attends to the
//    drafted nodes, whose masks it derives from the parents.
//  * tree_merge_kernel joins the partials and applies B^V.
//
// Precision: q~ and the probabilities are fp16 pairs (hi + lo, 22 bits), the
// codes, fp16 coefficients and queries are exact, sums and softmax statistics
// are float32.
#include <type_traits>

#include "entry.h"
#include "internal.h"

namespace dwkv {
namespace {

typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));
typedef __amdgpu_buffer_rsrc_t rsrc_t;

constexpr int D = kHeadDim;
constexpr int NW = kTreeWaves;           // waves per workgroup, two per SIMD
constexpr int TT = kTreeTile;            // tokens per tile
constexpr int kKRow = D + 8;             // halves per token row of the key code tile (16-byte pad: no bank conflicts)
constexpr float kUp = 6.0f;              // a moved reference leaves the largest probability at 2^6,
constexpr float kHead = 14.0f;           // and moves again when one exceeds 2^14: fp16 pairs hold both ends
constexpr int kBatches = 2;              // entry batches of 64 whose places a wave remembers for clearing

__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__device__ __forceinline__ rsrc_t make_rsrc(const void* base, int64_t bytes) {
  const uint32_t n = (uint32_t)min(max(bytes, (int64_t)0), (int64_t)0x7fffffff);
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, n, 0x00020000);
}

__device__ __forceinline__ int incl_max(int v) {   // running maximum over the lanes, v >= 0
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false));   // row_shr:1
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false));   // row_bcast:15
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false));   // row_bcast:31
  return v;
}

__device__ __forceinline__ f4 mfma_h(h8 a, h8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

template <bool BF>
__device__ __forceinline__ f4 mfma_q(u4v a, u4v b, f4 c) {
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
  else
    return mfma_h(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c);
}

__device__ __forceinline__ uint16_t h_bits(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
template <bool BF>
__device__ __forceinline__ uint16_t code_bits(float v) {   // v an int4 code: exact in both types
  return BF ? (uint16_t)(__builtin_bit_cast(uint32_t, v) >> 16) : h_bits(v);
}

// Place of a tile's token among the rows of the key code tile: score row r of
// token block b is token 8 (r / 4) + 4 b + r % 4, held at row 16 b + r, so that
// 16 lanes read 16 consecutive rows.
__device__ __forceinline__ int key_row(int t) { return 16 * ((t >> 2) & 1) + 4 * (t >> 3) + (t & 3); }

struct alignas(16) WaveTile {
  uint16_t k[TT * kKRow];                // key codes [token place][channel], zero between tiles
  uint16_t v[D * TT];                    // value codes [channel][token]
  float sk[TT], sv[TT];                  // residual scales of the tile's tokens (sv in units of 2^ex)
  uint8_t mark[64];
};

template <int RB>
struct Coef8 {                           // block scales of a tile, int8 coefficients
  alignas(16) uint16_t s[2][RB / 16][TT];
};
struct NoCoef8 {};

template <int NK, int NC, bool C8>
struct alignas(16) TreeSmem {
  static constexpr int RBP = 32 * NK, R = 16 * NC;
  u4v qf[4][NC][64];                     // query fragments: channels 32 s + 8 g + j
  u4v qt[2][NK][NC][64];                 // q~ fragments (hi, lo)
  float m[NW][R], l[NW][R];
  int ex[NW];
  float big;                             // largest |q~|
  union {
    WaveTile w[NW];
    float acc[NW][R][D + 4];             // the waves' sums, 128 columns at a time
  };
};
template <int NK, bool C8>
struct TreeSmem8 { typename std::conditional<C8, Coef8<32 * NK>, NoCoef8>::type c[C8 ? NW : 1]; };

// Sequence, row block, chunk and KV head of a workgroup.  Workgroups of one
// (chunk, KV head) follow each other on one XCD (consecutive workgroups go to
// the 8 XCDs in turn), so the row blocks share the chunk through its L2.
struct Item {
  int b, rb, h, c;                       // c == chunks: the drafted nodes
  int chunks, nrb;
  int t0, t1, n0, n;                     // tokens [t0, t1), nodes n0 .. n0 + n - 1 of the sequence
  int64_t part;                          // partial's index
};

__device__ __forceinline__ int seq_items(int T, int n, const TreeArgs& a, int& chunks, int& nrb) {
  chunks = T > 0 ? (T - 1) / a.split + 1 : 0;
  nrb = (n * a.group + a.rows - 1) / a.rows;
  return (chunks + 1) * nrb;
}

__device__ __forceinline__ Item find_item(const TreeArgs& a, int64_t x) {
  Item it;
  int64_t base = 0;
  const int H = a.n_kv_heads;
  if (a.wt.n_seq > 0) {
    it.b = 0;
    for (int i = 1; i < a.wt.n_seq; ++i)
      if (x >= (int64_t)a.wt.work[i] * H) it.b = i;
    base = a.wt.work[it.b];
    it.t0 = a.wt.tok[it.b];
    it.t1 = a.wt.tok[it.b + 1];
    it.n0 = a.wt.node[it.b];
    it.n = a.wt.node[it.b + 1] - it.n0;
  } else {                               // 64 sequences at a time
    const int lane = threadIdx.x & 63;
    for (int b0 = 0;; b0 += 64) {
      const int b = b0 + lane;
      int chunks, nrb, mine = 0;
      if (b < a.batch) mine = seq_items(a.cu[b + 1] - a.cu[b], a.cu_nodes[b + 1] - a.cu_nodes[b], a, chunks, nrb);
      int64_t end = mine;
      for (int d = 1; d < 64; d <<= 1) {
        const int64_t o = __shfl_up(end, d);
        if (lane >= d) end += o;
      }
      const unsigned long long in = __ballot(x < (base + end) * H);
      if (in) {
        const int w = __ffsll(in) - 1;
        base += __shfl(end - mine, w);
        it.b = b0 + w;
        break;
      }
      base += __shfl(end, 63);
      if (b0 + 64 >= a.batch) { it.b = a.batch - 1; break; }   // not reached: the grid ends with the items
    }
    it.t0 = a.cu[it.b];
    it.t1 = a.cu[it.b + 1];
    it.n0 = a.cu_nodes[it.b];
    it.n = a.cu_nodes[it.b + 1] - it.n0;
  }
  seq_items(it.t1 - it.t0, it.n, a, it.chunks, it.nrb);
  int64_t y = x - base * H;
  it.rb = (int)(y % it.nrb);
  y /= it.nrb;
  it.h = (int)(y % H);
  it.c = (int)(y / H);
  it.part = (base + (int64_t)it.c * it.nrb + it.rb) * H + it.h;
  return it;
}

// Ancestors of node `lane` of a sequence, itself included (bit j: node j), or
// 0 when it is absent; by pointer doubling over the wave.
__device__ __forceinline__ unsigned long long ancestors(const int32_t* parent, int n, int lane) {
  int p = lane < n ? parent[lane] : -2;
  bool bad = p < -1 || p >= lane;
  if (bad) p = -1;
  unsigned long long m = 1ull << lane;
  for (int d = 1; d < 64; d <<= 1) {
    const unsigned long long om = __shfl(m, max(p, 0));
    const int op = __shfl(p, max(p, 0)), ob = __shfl((int)bad, max(p, 0));
    if (p >= 0) {
      m |= om;
      bad |= ob != 0;
      p = op;
    }
  }
  return bad ? 0ull : m;
}

// Query element of row r (node r / G, member r % G), channel c, as float.
__device__ __forceinline__ float q_at(const TreeArgs& a, const Item& it, int r, int c) {
  const uint16_t* p = a.q + (int64_t)(it.n0 + r / a.group) * a.q_stride + (it.h * a.group + r % a.group) * D + c;
  return a.q_bf16 ? bf16_bits_to_float(*p) : half_bits_to_float(*p);
}

// The drafted nodes: a wave takes rows w, w + 8, ...; a lane takes node `lane`
// for the scores and channels 2 lane, 2 lane + 1 for the values.  Nodes a row
// does not see are skipped, not weighted with zero.
__device__ __forceinline__ void draft_item(const TreeArgs& a, const Item& it, int rows, float* part, int stride, int rbs) {
  const int wv = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const unsigned long long anc = ancestors(a.parent + it.n0, it.n, lane);
  const uint16_t* K = a.k_new + (int64_t)it.n0 * a.kv_stride + it.h * D;
  const uint16_t* V = a.v_new + (int64_t)it.n0 * a.kv_stride + it.h * D;
  const uint16_t* k = K + (int64_t)min(lane, it.n - 1) * a.kv_stride;
  for (int r0 = wv; r0 < rows; r0 += NW) {
    const int row = it.rb * rows + r0;
    float* o = part + (int64_t)r0 * stride;
    if (row >= it.n * a.group) continue;
    const unsigned long long see = __shfl(anc, row / a.group);
    float s = 0.f;
    for (int c = 0; c < D; c += 8) {
      const u4v w = *reinterpret_cast<const u4v*>(k + c);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s = __builtin_fmaf(half_bits_to_float(w[j] & 0xffff), q_at(a, it, row, c + 2 * j), s);
        s = __builtin_fmaf(half_bits_to_float(w[j] >> 16), q_at(a, it, row, c + 2 * j + 1), s);
      }
    }
    const bool mine = (see >> lane) & 1;
    s = mine ? s * a.qscale : -__builtin_inff();
    float m = s;
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    if (!(m > -__builtin_inff())) m = 0.f;                    // nothing seen, or -inf alone
    const float p = mine ? __builtin_amdgcn_exp2f(s - m) : 0.f;
    float l = p;
    for (int d = 32; d; d >>= 1) l += __shfl_xor(l, d);
    float o0 = 0.f, o1 = 0.f;
    for (unsigned long long left = see; left; left &= left - 1) {
      const int j = __ffsll(left) - 1;
      const float pj = __shfl(p, j);
      const uint32_t w = *reinterpret_cast<const uint32_t*>(V + (int64_t)j * a.kv_stride + 2 * lane);
      o0 = __builtin_fmaf(pj, half_bits_to_float(w & 0xffff), o0);
      o1 = __builtin_fmaf(pj, half_bits_to_float(w >> 16), o1);
    }
    *reinterpret_cast<float2*>(o + 2 * lane) = make_float2(o0, o1);
    for (int i = lane; i < rbs; i += 64) o[D + i] = 0.f;
    if (lane == 0) {
      o[D + rbs] = m;
      o[D + rbs + 1] = see ? l : -1.f;                        // -1: the node is absent
    }
  }
}

// Dequantized int8 coefficients, code * scale = hi + lo exactly (18 bits).
__device__ __forceinline__ void split8(const float (&v)[8], h8& hi, h8& lo) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    hi[j] = (_Float16)v[j];
    lo[j] = (_Float16)(v[j] - (float)hi[j]);
  }
}

__device__ __forceinline__ float byte_at(u2v w, int j) { return (float)(int8_t)(w[j >> 2] >> (8 * (j & 3))); }

template <int NK, int NC, bool BF, bool C8>
__global__ __launch_bounds__(64 * NW, 2) void tree_split_kernel(const TreeArgs a) {
  constexpr int R = 16 * NC, RBP = 32 * NK, NB = 2 * NK;
  __shared__ TreeSmem<NK, NC, C8> sm;
  __shared__ TreeSmem8<NK, C8> sm8;
  const int wv = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
  // consecutive workgroups of an XCD take consecutive items
  const int64_t per = (a.n_items + 7) / 8;
  const int64_t x = (int64_t)(blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if (x >= a.n_items) return;
  const Item it = find_item(a, x);
  const int rb = a.rb, nb = rb / 16, rows_left = it.n * a.group - it.rb * R;
  const int stride = D + rb + 4;
  float* part = a.part + it.part * R * stride;
  if (it.c == it.chunks) {
    draft_item(a, it, R, part, stride, rb);
    return;
  }

  // ---- query fragments, and q~ = B^K q as fp16 pairs ---------------------------
  for (int i = threadIdx.x; i < 4 * NC * 64; i += 64 * NW) {
    const int ln = i & 63, n = (i >> 6) % NC, s = (i >> 6) / NC, r = 16 * n + (ln & 15);
    u4v w = {0, 0, 0, 0};
    if (r < rows_left) {
      const int row = it.rb * R + r;
      const int p = a.parent[it.n0 + row / a.group];
      if (p >= -1 && p < row / a.group)
        w = *reinterpret_cast<const u4v*>(a.q + (int64_t)(it.n0 + row / a.group) * a.q_stride +
                                          (it.h * a.group + row % a.group) * D + 32 * s + 8 * (ln >> 4));
    }
    sm.qf[s][n][ln] = w;
  }
  if (threadIdx.x == 0) sm.big = 0.f;
  __syncthreads();
  const uint16_t* bk = a.basis + (int64_t)it.b * a.basis_b_stride + (int64_t)(it.h * 2) * rb * D;
  {
    const int tiles = nb * NC;
    f4 q[(NB * NC + NW - 1) / NW];
    float big = 0.f;
#pragma unroll
    for (int u = 0; u < (NB * NC + NW - 1) / NW; ++u) {
      const int tile = wv + NW * u, blk = tile / NC, n = tile % NC;
      f4 c = {0.f, 0.f, 0.f, 0.f};
      if (tile < tiles) {
        for (int s = 0; s < 4; ++s) {
          const u4v w = sm.qf[s][n][lane];             // channels 32 s + 8 g + j
          const u4v bw = *reinterpret_cast<const u4v*>(bk + (16 * blk + col) * D + 32 * s + 8 * g);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint16_t qb = (uint16_t)(w[j >> 1] >> (16 * (j & 1))), bb = (uint16_t)(bw[j >> 1] >> (16 * (j & 1)));
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(half_bits_to_float(bb), BF ? bf16_bits_to_float(qb) : half_bits_to_float(qb), c, 0, 0, 0);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        c[i] *= a.qscale;
        const float m = fabsf(c[i]);
        if (m < __builtin_inff()) big = fmaxf(big, m);
      }
      q[u] = c;
    }
    // |q~| beyond fp16 is scaled down for the whole workgroup (scores stay float32)
    atomicMax(reinterpret_cast<int*>(&sm.big), __builtin_bit_cast(int, big));
    __syncthreads();
    const int down = max(0, __builtin_amdgcn_frexp_expf(sm.big) - 15);
    const float f = __builtin_ldexpf(1.f, -down);
#pragma unroll
    for (int u = 0; u < (NB * NC + NW - 1) / NW; ++u) {
      const int tile = wv + NW * u, blk = tile / NC, n = tile % NC;
      if (tile >= NB * NC) continue;
      h4 hi, lo;                                       // basis rows 16 blk + 4 g + i, zero past r_b
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float v = q[u][i] * f;
        hi[i] = (_Float16)v;
        lo[i] = (_Float16)(v - (float)hi[i]);
      }
      const int ln = 16 * (2 * (blk & 1) + (g >> 1)) + col;
      reinterpret_cast<h4*>(&sm.qt[0][blk >> 1][n][ln])[g & 1] = hi;
      reinterpret_cast<h4*>(&sm.qt[1][blk >> 1][n][ln])[g & 1] = lo;
    }
  }
  const int down = max(0, __builtin_amdgcn_frexp_expf(sm.big) - 15);
  const float up = __builtin_ldexpf(1.f, down), fdn = __builtin_ldexpf(1.f, -down);

  // ---- the chunk's streams -----------------------------------------------------
  const int c0 = it.t0 + it.c * a.split, c1 = it.t1 - c0 > a.split ? c0 + a.split : it.t1, tb = c0 & ~15;
  const int ntile = (c1 - tb + TT - 1) / TT;
  const int64_t T = a.T, T16 = (T + 15) / 16 * 16;
  const int esz = C8 ? 1 : 2;
  const uint8_t* ckp = reinterpret_cast<const uint8_t*>(a.coef_k) + (int64_t)it.h * T16 * rb * esz;
  const uint8_t* cvp = reinterpret_cast<const uint8_t*>(a.coef_v) + (int64_t)it.h * T16 * rb * esz;
  const rsrc_t rk = make_rsrc(ckp + (int64_t)tb * rb * esz, (T16 - tb) * rb * esz);
  const rsrc_t rv = make_rsrc(cvp + (int64_t)tb * rb * esz, (T16 - tb) * rb * esz);
  const uint32_t* off = a.off + (int64_t)it.h * (T + 1);
  const uint32_t ec0 = off[c0];
  const uint8_t* idx[2] = {a.idx_k + (int64_t)it.h * a.res_stride, a.idx_v + (int64_t)it.h * a.res_stride};
  const uint8_t* val[2] = {a.val_k + (int64_t)it.h * (a.res_stride / 2), a.val_v + (int64_t)it.h * (a.res_stride / 2)};
  const int64_t eroom = a.res_stride - (int64_t)ec0;   // entries of the slab from the chunk on (ec0 is even)
  const rsrc_t ri[2] = {make_rsrc(idx[0] + (eroom > 0 ? ec0 : 0), eroom), make_rsrc(idx[1] + (eroom > 0 ? ec0 : 0), eroom)};
  const rsrc_t rw[2] = {make_rsrc(val[0] + (eroom > 0 ? ec0 / 2 : 0), eroom / 2), make_rsrc(val[1] + (eroom > 0 ? ec0 / 2 : 0), eroom / 2)};
  const uint16_t* sk = a.scale_k + (int64_t)it.h * T;
  const uint16_t* sv = a.scale_v + (int64_t)it.h * T;

  WaveTile& w = sm.w[wv];
  for (int i = lane; i < (int)((sizeof(w.k) + sizeof(w.v)) / 16); i += 64) reinterpret_cast<u4v*>(&w)[i] = u4v{0, 0, 0, 0};
  __syncthreads();                       // q~ and the fragments are whole

  u4v qf[4][NC], qt[2][NK][NC];
#pragma unroll
  for (int n = 0; n < NC; ++n) {
#pragma unroll
    for (int s = 0; s < 4; ++s) qf[s][n] = sm.qf[s][n][lane];
#pragma unroll
    for (int s = 0; s < NK; ++s) {
      qt[0][s][n] = sm.qt[0][s][n][lane];
      qt[1][s][n] = sm.qt[1][s][n][lane];
    }
  }
  f4 acc_a[NB][NC], acc_r[D / 16][NC];   // a~ and the residual channels: (channel 4 g + i of the block, row col)
  float m[NC], l[NC];
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    m[n] = l[n] = 0.f;
#pragma unroll
    for (int k = 0; k < NB; ++k) acc_a[k][n] = f4{0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < D / 16; ++k) acc_r[k][n] = f4{0, 0, 0, 0};
  }
  bool first = true;
  int ex = -24;                          // |s^V| <= 2^ex of the tiles so far

  for (int j = wv; j < ntile; j += NW) {
    const int t0 = tb + j * TT, rel = j * TT;          // tile's first token; relative to tb
    const bool edge = t0 < c0 || t0 + TT > c1;
    // ---- offsets and scales, one lane per token
    const int tl = t0 + (lane & 31);
    const uint32_t oa = off[min(max(tl, c0), c1)] - ec0, ob = off[min(max(tl + 1, c0), c1)] - ec0;
    const bool in = tl >= c0 && tl < c1;
    float fk = 0.f, fv = 0.f;
    if (in && ob > oa) {
      fk = half_bits_to_float(sk[tl]);
      fv = half_bits_to_float(sv[tl]);
    }
    const float inf = __builtin_inff();
    const bool odd_k = !(fabsf(fk) < inf), odd_v = !(fabsf(fv) < inf);
    if (__ballot(!odd_v && fabsf(fv) > __builtin_ldexpf(1.f, ex))) {      // rare: larger value scales
      int e = !odd_v && fv != 0.f ? __builtin_amdgcn_frexp_expf(fv) : -24;
      for (int d = 32; d; d >>= 1) e = max(e, __shfl_xor(e, d));
      const float fall = __builtin_ldexpf(1.f, ex - e);
      ex = e;
#pragma unroll
      for (int k = 0; k < D / 16; ++k)
#pragma unroll
        for (int n = 0; n < NC; ++n) acc_r[k][n] *= fall;
    }
    // a scale that is not finite goes with its entries into the code tiles
    if (lane < 32) {
      w.sk[lane] = odd_k ? a.qscale : fk * a.qscale;
      w.sv[lane] = odd_v ? 1.f : __builtin_ldexpf(fv, -ex);
    }
    // ---- entries into the code tiles, 64 at a time
    const uint32_t e0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)oa);
    const uint32_t e1 = (uint32_t)__builtin_amdgcn_readlane((int)ob, 31);
    const uint32_t n = e1 > e0 ? min(e1 - e0, (uint32_t)(TT * D)) : 0u;
    const bool odd = __ballot(odd_k || odd_v) != 0;
    const uint32_t odd_tokens = (uint32_t)__ballot(odd_v);   // lanes 32 .. 63 repeat the first 32
    uint32_t place[kBatches];
    int carry = 0;
#pragma unroll 1
    for (uint32_t b0 = 0, it_b = 0; b0 < n; b0 += 64, ++it_b) {
      const uint32_t e = e0 + b0 + lane;
      const uint32_t ck = __builtin_amdgcn_raw_buffer_load_b8(ri[0], e, 0, 0), cv = __builtin_amdgcn_raw_buffer_load_b8(ri[1], e, 0, 0);
      const uint32_t vk = __builtin_amdgcn_raw_buffer_load_b8(rw[0], e >> 1, 0, 0), vv = __builtin_amdgcn_raw_buffer_load_b8(rw[1], e >> 1, 0, 0);
      w.mark[lane] = 0;
      wave_lds_sync();
      if (lane < 32 && ob > oa && oa - e0 >= b0 && oa - e0 < b0 + 64) w.mark[oa - e0 - b0] = (uint8_t)(lane + 1);
      wave_lds_sync();
      const int tok = max(incl_max((int)w.mark[lane]), carry);
      carry = __builtin_amdgcn_readlane(tok, 63);
      uint32_t at = 0xffffffffu;
      const bool live = b0 + lane < n && tok > 0;
      if (live) {
        const int t = tok - 1;
        const uint32_t pk = key_row(t) * kKRow + (ck & (D - 1)), pv = (cv & (D - 1)) * TT + t;
        at = pk | pv << 16;
        float fck = (float)entry_code(vk, e), fcv = (float)entry_code(vv, e);
        uint16_t wk = code_bits<BF>(fck), wv16 = h_bits(fcv);
        if (odd) {
          const float tk = half_bits_to_float(sk[t0 + t]), tv = half_bits_to_float(sv[t0 + t]);
          if (!(fabsf(tk) < inf)) wk = BF ? (uint16_t)(__builtin_bit_cast(uint32_t, fck * tk) >> 16) : h_bits(fck * tk);
          if (!(fabsf(tv) < inf)) wv16 = h_bits(fcv * tv);
        }
        w.k[pk] = wk;
        w.v[pv] = wv16;
      }
      if (it_b == 0) place[0] = at;
      else if (it_b == 1) place[1] = at;
    }
    wave_lds_sync();

    // ---- scores: (token 8 g + 4 b + i, row col)
    float ks[8], vs[8];
    {
      const f4 s0 = *reinterpret_cast<const f4*>(&w.sk[8 * g]), s1 = *reinterpret_cast<const f4*>(&w.sk[8 * g + 4]);
      const f4 v0 = *reinterpret_cast<const f4*>(&w.sv[8 * g]), v1 = *reinterpret_cast<const f4*>(&w.sv[8 * g + 4]);
#pragma unroll
      for (int i = 0; i < 4; ++i) { ks[i] = s0[i]; ks[4 + i] = s1[i]; vs[i] = v0[i]; vs[4 + i] = v1[i]; }
    }
    if constexpr (C8) {
      if (lane < 32) {
        const int64_t tc = min((int64_t)(t0 + lane), T - 1);
        for (int s = 0; s < nb; ++s) {
          sm8.c[wv].s[0][s][lane] = a.cscale_k[((int64_t)it.h * nb + s) * T + tc];
          sm8.c[wv].s[1][s][lane] = a.cscale_v[((int64_t)it.h * nb + s) * T + tc];
        }
      }
      wave_lds_sync();
    }
    float p[2][NC][4];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int tk = 8 * (col >> 2) + 4 * b + (col & 3);           // token of score row `col`
      const int tr = rel + tk;
      f4 sb[NC], sr[NC];
#pragma unroll
      for (int n2 = 0; n2 < NC; ++n2) {
        const float c = -m[n2] * fdn;
        sb[n2] = f4{c, c, c, c};
        sr[n2] = f4{0, 0, 0, 0};
      }
#pragma unroll
      for (int s = 0; s < NK; ++s) {
        if (32 * s < rb) {
          const bool have = 32 * s + 8 * g < rb;
          if constexpr (C8) {
            u2v cw = {0, 0};
            float v[8] = {};
            if (have) {
              cw = __builtin_amdgcn_raw_buffer_load_b64(rk, (((tr >> 4) * nb + 2 * s + (g >> 1)) * 16 + (tr & 15)) * 16 + 8 * (g & 1), 0, 0);
              const float sc = half_bits_to_float(sm8.c[wv].s[0][2 * s + (g >> 1)][tk]);
#pragma unroll
              for (int e = 0; e < 8; ++e) v[e] = byte_at(cw, e) * sc;
            }
            h8 hi, lo;
            split8(v, hi, lo);
#pragma unroll
            for (int n2 = 0; n2 < NC; ++n2) {
              sb[n2] = mfma_h(hi, __builtin_bit_cast(h8, qt[0][s][n2]), sb[n2]);
              sb[n2] = mfma_h(hi, __builtin_bit_cast(h8, qt[1][s][n2]), sb[n2]);
              sb[n2] = mfma_h(lo, __builtin_bit_cast(h8, qt[0][s][n2]), sb[n2]);
            }
          } else {
            u4v cw = {0, 0, 0, 0};
            if (have) cw = __builtin_amdgcn_raw_buffer_load_b128(rk, (((tr >> 4) * (rb / 8) + 4 * s + g) * 128 + (tr & 15) * 8) * 2, 0, 0);
            const h8 av = __builtin_bit_cast(h8, cw);
#pragma unroll
            for (int n2 = 0; n2 < NC; ++n2) {
              sb[n2] = mfma_h(av, __builtin_bit_cast(h8, qt[0][s][n2]), sb[n2]);
              sb[n2] = mfma_h(av, __builtin_bit_cast(h8, qt[1][s][n2]), sb[n2]);
            }
          }
        }
      }
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const u4v kc = *reinterpret_cast<const u4v*>(&w.k[(16 * b + col) * kKRow + 32 * s + 8 * g]);
#pragma unroll
        for (int n2 = 0; n2 < NC; ++n2) sr[n2] = mfma_q<BF>(kc, qf[s][n2], sr[n2]);
      }
#pragma unroll
      for (int n2 = 0; n2 < NC; ++n2)
#pragma unroll
        for (int i = 0; i < 4; ++i) p[b][n2][i] = __builtin_fmaf(ks[4 * b + i], sr[n2][i], down ? sb[n2][i] * up : sb[n2][i]);
    }
    if (edge) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = t0 + 8 * g + 4 * b + i;
          if (t < c0 || t >= c1)
#pragma unroll
            for (int n2 = 0; n2 < NC; ++n2) p[b][n2][i] = -inf;
        }
    }
    // ---- the reference moves for the first tile and when a score exceeds it by far
    float mx[NC];
    bool move = first;
#pragma unroll
    for (int n2 = 0; n2 < NC; ++n2) {
      mx[n2] = fmaxf(fmaxf(fmaxf(p[0][n2][0], p[0][n2][1]), fmaxf(p[0][n2][2], p[0][n2][3])),
                     fmaxf(fmaxf(p[1][n2][0], p[1][n2][1]), fmaxf(p[1][n2][2], p[1][n2][3])));
      move = move || mx[n2] > kHead;
    }
    if (__ballot(move)) {
#pragma unroll
      for (int n2 = 0; n2 < NC; ++n2) {
        float c = fmaxf(mx[n2], __shfl_xor(mx[n2], 16));
        c = fmaxf(c, __shfl_xor(c, 32));
        const float by = (first ? c > -inf : c > kHead) ? c - kUp : 0.f;
        const float fall = first ? 0.f : __builtin_amdgcn_exp2f(-by);
        m[n2] += by;
        l[n2] *= fall;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) p[b][n2][i] -= by;
        if (!first) {
#pragma unroll
          for (int k = 0; k < NB; ++k) acc_a[k][n2] *= fall;
#pragma unroll
          for (int k = 0; k < D / 16; ++k) acc_r[k][n2] *= fall;
        }
      }
      first = false;
    }
    // ---- probabilities as fp16 pairs, plain and times the value scales
    h8 ph[NC], pl[NC], rh[NC], rl[NC];
#pragma unroll
    for (int n2 = 0; n2 < NC; ++n2) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = __builtin_amdgcn_exp2f(p[e >> 2][n2][e & 3]);
        sum += v;
        ph[n2][e] = (_Float16)v;
        pl[n2][e] = (_Float16)(v - (float)ph[n2][e]);
        const float u = v * vs[e];
        rh[n2][e] = (_Float16)u;
        rl[n2][e] = (_Float16)(u - (float)rh[n2][e]);
      }
      l[n2] += sum;
      if (odd_tokens) {                  // an infinite entry meets positive numbers only
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if ((odd_tokens >> (8 * g + e)) & 1) {
            rh[n2][e] = rh[n2][e] > (_Float16)0x1p-14f ? rh[n2][e] : (_Float16)0x1p-14f;
            rl[n2][e] = (_Float16)0x1p-14f;
          }
      }
    }
    // ---- values: channel blocks of the basis, then of the residual
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      if (16 * k < rb) {
        if constexpr (C8) {
          const u2v cw = __builtin_amdgcn_raw_buffer_load_b64(rv, ((((rel >> 4) + (g >> 1)) * rb + 16 * k + col) * 16) + 8 * (g & 1), 0, 0);
          const u4v sw = *reinterpret_cast<const u4v*>(&sm8.c[wv].s[1][k][8 * g]);
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = byte_at(cw, e) * half_bits_to_float((uint16_t)(sw[e >> 1] >> (16 * (e & 1))));
          if (edge) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (t0 + 8 * g + e < c0 || t0 + 8 * g + e >= c1) v[e] = 0.f;
          }
          h8 hi, lo;
          split8(v, hi, lo);
#pragma unroll
          for (int n2 = 0; n2 < NC; ++n2) {
            acc_a[k][n2] = mfma_h(hi, ph[n2], acc_a[k][n2]);
            acc_a[k][n2] = mfma_h(hi, pl[n2], acc_a[k][n2]);
            acc_a[k][n2] = mfma_h(lo, ph[n2], acc_a[k][n2]);
          }
        } else {
          h8 av = __builtin_bit_cast(h8, __builtin_amdgcn_raw_buffer_load_b128(rv, (((rel >> 3) + g) * rb + 16 * k + col) * 16, 0, 0));
          if (edge) {                    // tokens outside the chunk may hold anything
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (t0 + 8 * g + e < c0 || t0 + 8 * g + e >= c1) av[e] = (_Float16)0.f;
          }
#pragma unroll
          for (int n2 = 0; n2 < NC; ++n2) {
            acc_a[k][n2] = mfma_h(av, ph[n2], acc_a[k][n2]);
            acc_a[k][n2] = mfma_h(av, pl[n2], acc_a[k][n2]);
          }
        }
      }
    }
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      const h8 av = __builtin_bit_cast(h8, *reinterpret_cast<const u4v*>(&w.v[(16 * k + col) * TT + 8 * g]));
#pragma unroll
      for (int n2 = 0; n2 < NC; ++n2) {
        acc_r[k][n2] = mfma_h(av, rh[n2], acc_r[k][n2]);
        acc_r[k][n2] = mfma_h(av, rl[n2], acc_r[k][n2]);
      }
    }
    // ---- the code tiles go back to zero
    wave_lds_sync();
    if (n > 64 * kBatches) {
      for (int i = lane; i < (int)((sizeof(w.k) + sizeof(w.v)) / 16); i += 64) reinterpret_cast<u4v*>(&w)[i] = u4v{0, 0, 0, 0};
    } else {
      if (n > 0 && place[0] != 0xffffffffu) { w.k[place[0] & 0xffff] = 0; w.v[place[0] >> 16] = 0; }
      if (n > 64 && place[1] != 0xffffffffu) { w.k[place[1] & 0xffff] = 0; w.v[place[1] >> 16] = 0; }
    }
    wave_lds_sync();
  }

  // ---- join the waves: common reference per row, then sums in wave order -----------
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    l[n] += __shfl_xor(l[n], 16);
    l[n] += __shfl_xor(l[n], 32);
    if (g == 0) {
      sm.m[wv][16 * n + col] = first ? -__builtin_inff() : m[n];
      sm.l[wv][16 * n + col] = l[n];
    }
  }
  __syncthreads();                       // the code tiles are done with
  float mine[NC];
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    float ms = -__builtin_inff();
    for (int u = 0; u < NW; ++u) ms = fmaxf(ms, sm.m[u][16 * n + col]);
    mine[n] = first ? 0.f : __builtin_amdgcn_exp2f(m[n] - ms);
  }
  const float rex = __builtin_ldexpf(1.f, ex);
#pragma unroll
  for (int k = 0; k < D / 16; ++k)
#pragma unroll
    for (int n = 0; n < NC; ++n)
      *reinterpret_cast<f4*>(&sm.acc[wv][16 * n + col][16 * k + 4 * g]) = acc_r[k][n] * (mine[n] * rex);
  __syncthreads();
  for (int i = threadIdx.x; i < R * D; i += 64 * NW) {
    const int r = i / D, c = i % D;
    float s = 0.f;
    for (int u = 0; u < NW; ++u) s += sm.acc[u][r][c];
    if (r < rows_left) part[(int64_t)r * stride + c] = s;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < NB; ++k)
#pragma unroll
    for (int n = 0; n < NC; ++n)
      *reinterpret_cast<f4*>(&sm.acc[wv][16 * n + col][16 * k + 4 * g]) = acc_a[k][n] * mine[n];
  __syncthreads();
  for (int i = threadIdx.x; i < R * rb; i += 64 * NW) {
    const int r = i / rb, c = i % rb;
    float s = 0.f;
    for (int u = 0; u < NW; ++u) s += sm.acc[u][r][c];
    if (r < rows_left) part[(int64_t)r * stride + D + c] = s;
  }
  if (threadIdx.x < R && (int)threadIdx.x < rows_left) {
    const int r = threadIdx.x;
    float ms = -__builtin_inff(), ls = 0.f;
    for (int u = 0; u < NW; ++u) ms = fmaxf(ms, sm.m[u][r]);
    for (int u = 0; u < NW; ++u)
      if (sm.m[u][r] > -__builtin_inff()) ls += sm.l[u][r] * __builtin_amdgcn_exp2f(sm.m[u][r] - ms);
    part[(int64_t)r * stride + D + rb] = ms;
    part[(int64_t)r * stride + D + rb + 1] = ls;
  }
}

// One workgroup per (node and member row of 4 rows, sequence and KV head): joins
// the partials of its rows, applies B^V.  grid (row quads of the longest sequence, Hkv, B)
constexpr int kMR = 4;
__global__ __launch_bounds__(128) void tree_merge_kernel(const TreeArgs a) {
  __shared__ float as[kMR][128];
  const int b = blockIdx.z, h = blockIdx.y, c = threadIdx.x, H = a.n_kv_heads, rb = a.rb;
  int64_t base = 0;
  int t0, t1, n0, n;
  if (a.wt.n_seq > 0) {
    base = a.wt.work[b];
    t0 = a.wt.tok[b], t1 = a.wt.tok[b + 1], n0 = a.wt.node[b], n = a.wt.node[b + 1] - n0;
  } else {
    const int lane = threadIdx.x & 63;
    for (int i = lane; i < b; i += 64) {
      int ch, nr;
      base += seq_items(a.cu[i + 1] - a.cu[i], a.cu_nodes[i + 1] - a.cu_nodes[i], a, ch, nr);
    }
    for (int d = 32; d; d >>= 1) base += __shfl_xor(base, d);
    t0 = a.cu[b], t1 = a.cu[b + 1], n0 = a.cu_nodes[b], n = a.cu_nodes[b + 1] - n0;
  }
  int chunks, nrb;
  seq_items(t1 - t0, n, a, chunks, nrb);
  const int r0 = blockIdx.x * kMR, rows = n * a.group;
  if (r0 >= rows) return;
  const int stride = D + rb + 4, block = r0 / a.rows;         // a.rows is a multiple of kMR
  const float* p0 = a.part + ((base + block) * H + h) * a.rows * stride + (int64_t)(r0 % a.rows) * stride;
  const int64_t step = (int64_t)nrb * H * a.rows * stride;    // to the next chunk's partial
  float out[kMR];
#pragma unroll
  for (int r = 0; r < kMR; ++r) {
    out[r] = 0.f;
    as[r][c] = 0.f;
    if (r0 + r >= rows) continue;
    const float* p = p0 + (int64_t)r * stride;
    float ms = -__builtin_inff();
    bool absent = false;
    for (int s = 0; s <= chunks; ++s) {
      const float l = p[s * step + D + rb + 1];
      if (l < 0.f) absent = true;
      if (!(l == 0.f)) ms = fmaxf(ms, p[s * step + D + rb]);
    }
    if (absent) continue;
    float l = 0.f, o = 0.f, av = 0.f;
    for (int s = 0; s <= chunks; ++s) {
      const float* ps = p + s * step;
      const float ls = ps[D + rb + 1];
      if (ls == 0.f) continue;
      const float wt = __builtin_amdgcn_exp2f(ps[D + rb] - ms);
      l = __builtin_fmaf(wt, ls, l);
      o = __builtin_fmaf(wt, ps[c], o);
      if (c < rb) av = __builtin_fmaf(wt, ps[D + c], av);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    out[r] = o * inv;
    as[r][c] = av * inv;
  }
  __syncthreads();
  const uint16_t* bv = a.basis + (int64_t)b * a.basis_b_stride + (int64_t)(h * 2 + 1) * rb * D;
  for (int i = 0; i < rb; ++i) {
    const float v = half_bits_to_float(bv[i * D + c]);
#pragma unroll
    for (int r = 0; r < kMR; ++r) out[r] = __builtin_fmaf(as[r][i], v, out[r]);
  }
#pragma unroll
  for (int r = 0; r < kMR; ++r)
    if (r0 + r < rows)
      a.out[((int64_t)(n0 + (r0 + r) / a.group) * a.n_q_heads + h * a.group + (r0 + r) % a.group) * D + c] = out[r];
}

template <int NK, int NC, bool BF>
void launch_c(const TreeArgs& a, dim3 grid, hipStream_t s) {
  if (a.c8) hipLaunchKernelGGL((tree_split_kernel<NK, NC, BF, true>), grid, dim3(64 * NW), 0, s, a);
  else hipLaunchKernelGGL((tree_split_kernel<NK, NC, BF, false>), grid, dim3(64 * NW), 0, s, a);
}

template <int NK>
void launch_k(const TreeArgs& a, dim3 grid, hipStream_t s) {
  if (NK > 2 || a.rows == 16) {
    if (a.q_bf16) launch_c<NK, 1, true>(a, grid, s);
    else launch_c<NK, 1, false>(a, grid, s);
  } else if constexpr (NK <= 2) {
    if (a.q_bf16) launch_c<NK, 2, true>(a, grid, s);
    else launch_c<NK, 2, false>(a, grid, s);
  }
}

}  // namespace

hipError_t launch_tree(const TreeArgs& a, int max_rows, hipStream_t s) {
  const dim3 grid((unsigned)((a.n_items + 7) / 8 * 8));
  if (a.rb <= 32) launch_k<1>(a, grid, s);
  else if (a.rb <= 64) launch_k<2>(a, grid, s);
  else launch_k<4>(a, grid, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(tree_merge_kernel, dim3((max_rows + kMR - 1) / kMR, a.n_kv_heads, a.batch), dim3(128), 0, s, a);
  return hipGetLastError();
}

}  // namespace dwkv
