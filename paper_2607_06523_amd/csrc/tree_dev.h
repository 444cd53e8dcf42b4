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
//    block of 32 rows), its waves taking the chunk's 32-token tiles in turn.
//    Scores come out transposed, tokens down the accumulator and rows across,
//    which is the operand layout the value products read: probabilities never
//    leave the registers.  A tile's tokens are dealt to the score rows so that
//    eight consecutive scores of a lane are eight consecutive tokens, one
//    value block.  All products are 32x32x16: beside one of them, unlike a pair
//    of 16x16x32, the vector unit goes on (four 16x16x32 and twelve vector
//    instructions of each of two waves take 93 ns, the same work in two 32x32x16
//    69, the products alone 72 and 71).
//  * one more workgroup per (sequence, KV head, row block) attends to the
//    drafted nodes, whose masks it derives from the parents.
//  * tree_merge_kernel joins the partials and applies B^V.
//
// Precision: q~, the probabilities and their products with the value scales are fp16
// pairs (hi + lo, 22 bits) in units of the row's own (row_down, kUp, rs); the codes,
// fp16 coefficients and queries are exact, sums and softmax statistics are float32.
// One half alone would cost 2^-11 of a score or probability, fifty times what the
// decode keeps.
//
// Measured at 65536 tokens, r_b 48, G 4, 8 KV heads, mean rank 1.9 (110 MB): 64 nodes
// 175 us with the merge.  The pairs and the dense code tiles make it 38 products per
// tile and 32 rows, 163 GFLOP in all, 0.93 PFLOP/s; the matrix cores are busy 45%
// of the compute units' cycles and the clock falls to 1.9 GHz, so that a kernel with
// 11% fewer cycles took the same time.  8 nodes: 41 us, 2.65 TB/s.  Traced, where
// launches do not overlap: 37 for this pass, of them 4 until a workgroup's q~ is
// there and 4 to join its waves, most of the rest its 9 tiles per wave, and 7
// for the merge.  A scale of its own for every row, in place of one per workgroup or
// wave, is 2 to 4% of these times.  Blocks of 64 rows (each tile's codes scattered
// half as often) do not fit the registers: the loop's spills wait for its loads.
#pragma once
#include "entry.h"
#include "internal.h"

namespace dwkv {
namespace {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));
typedef __amdgpu_buffer_rsrc_t rsrc_t;

constexpr int D = kHeadDim;
constexpr int TT = kTreeTile;            // tokens per tile
constexpr int R = kTreeRows;             // rows of a workgroup
constexpr int kKRow = D + 8;             // halves per token row of the key code tile (16-byte pad: no bank conflicts)
constexpr int kWaitVmcnt0 = 0x0F70;      // s_waitcnt immediate: vmcnt(0) only
// A moved reference leaves the largest probability at 2^kUp and moves again when one
// exceeds 2^kHead, the most that fp16 holds: 22 bits down to 2^-12 of the largest,
// below it a grid of 2^-33 of the largest.  With 12 for kUp references move often
// enough to cost 3 to 6% (16 int8 sequences 219 us, 208 at 9 and at 6).
constexpr float kUp = 9.0f;
constexpr float kHead = 15.5f;
constexpr float kFull = 15.5f;           // largest exponent of a scaled residual weight
constexpr int kMost = 40;                // largest exponent of their scale: also that of rows without one
constexpr int kNoScale = -64;            // ex before the first value scale: lim is kHead then, whatever rs is

__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__device__ __forceinline__ rsrc_t make_rsrc(const void* base, int64_t bytes) {
  const uint32_t n = (uint32_t)min(max(bytes, (int64_t)0), (int64_t)1 << 30);   // a chunk is far shorter
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

__device__ __forceinline__ f16v mfma_h(h8 a, h8 b, f16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

template <bool BF>
__device__ __forceinline__ f16v mfma_q(u4v a, u4v b, f16v c) {
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
  else
    return mfma_h(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c);
}

__device__ __forceinline__ uint16_t h_bits(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
template <bool BF>
__device__ __forceinline__ uint16_t code_bits(float v) {   // v an int4 code: exact in both types
  return BF ? (uint16_t)(__builtin_bit_cast(uint32_t, v) >> 16) : h_bits(v);
}

// Score row of a tile's token.  Accumulator register 4 a + i of lane half h is score
// row 8 a + 4 h + i; with these rows it is token 16 (a / 2) + 8 h + 4 (a % 2) + i, so
// that registers 8 u .. 8 u + 7 are tokens 16 u + 8 h .. + 7, the u-th 16-deep step of
// the value products.
__device__ __forceinline__ int key_row(int t) { return 16 * (t >> 4) + 8 * ((t >> 2) & 1) + 4 * ((t >> 3) & 1) + (t & 3); }
__device__ __forceinline__ int row_token(int r) { return 16 * (r >> 4) + 8 * ((r >> 2) & 1) + 4 * ((r >> 3) & 1) + (r & 3); }

// Binary places by which a row's q~ is scaled down, or up where negative, so that
// its largest number `big` is between 2^14 and 2^15: pairs hold it to 22 bits, and
// numbers 2^17 times smaller as well.  A row has its own scale, and nothing of
// the rows beside it.  2^48 is enough: what pairs lose then is below 2^-50 of a
// score with the largest coefficients.
__device__ __forceinline__ int row_down(float big) { return max(big > 0.f ? __builtin_amdgcn_frexp_expf(big) - 15 : 0, -48); }

// Place of (channel, token) in the value code tile: a channel's four 8-token
// pieces are dealt by channel, so that 16 lanes reading the same piece of 16
// channels touch every bank once.
__device__ __forceinline__ uint32_t value_place(uint32_t c, uint32_t t) { return c * TT + (((t >> 3) ^ ((c >> 2) & 3)) << 3) + (t & 7); }

// Lanes without an entry write past the ends of k and v and of mark's first half:
// no branch keeps them out.
struct alignas(16) WaveTile {
  uint16_t k[TT * kKRow + 8];            // key codes [token place][channel], zero between tiles
  uint16_t v[D * TT + 8];                // value codes (value_place)
  float sk[TT], sv[TT];                  // residual scales of the tile's tokens
  uint8_t mark[128];
};
constexpr uint32_t kNoKey = TT * kKRow, kNoValue = D * TT;

// Smem of the drafted nodes' workgroups.
struct alignas(16) DraftSmem {
  float q[R][D];
  uint16_t v[DWKV_MAX_TREE_NODES][D];
};

// Waves of a workgroup: two per SIMD, or one where the sums and fragments of wide
// bases take more than half its registers.
template <int NB>
constexpr int kWaves = NB > 4 ? 4 : 8;

template <int NB, bool C8>
struct alignas(16) TreeSmem {
  static constexpr int NW = kWaves<NB>;
  float m[NW][R], l[NW][R];              // statistics; during the tiles m holds a row's largest residual weight
  uint32_t odd[D];                       // channels with entries of value scales that are not finite: bits +inf, -inf, NaN
  float big[R];                          // largest finite |q~| of a row
  alignas(16) uint16_t vs[C8 ? NW : 1][C8 ? NB : 1][C8 ? TT : 8];   // value block scales of a tile (int8)
  union {
    struct {
      WaveTile w[NW];
      u4v qf[8][64];                     // query fragments: channels 16 s + 8 h + j of row lane % 32
      u4v qt[2][NB][64];                 // q~ fragments (hi, lo)
    };
    float acc[NW][R][D + 4];             // the waves' sums, 128 columns at a time
    DraftSmem d;
  };
};

// Sequence, row block, chunk and KV head of a workgroup.
struct Item {
  int b, rb, h, c;                       // c == chunks: the drafted nodes
  int chunks, nrb;                       // nrb == 0: no sequence has this item
  int t0, t1, n0, n;                     // tokens [t0, t1), nodes n0 .. n0 + n - 1 of the sequence
  int64_t part;                          // partial's index
};

__device__ __forceinline__ void seq_items(int T, int n, const TreeArgs& a, int& chunks, int& nrb) {
  chunks = T > 0 ? (T - 1) / a.split + 1 : 0;
  nrb = (n * a.group + R - 1) / R;
}

// Workgroups go to the 8 XCDs in turn.  The row blocks of one (chunk, KV head)
// follow each other on one XCD, so that they share the chunk through its L2:
// workgroup w is row block (w / 8) % max_nrb of pair w % 8 + 8 (w / 8 / max_nrb),
// the pairs (chunk, KV head) counted over the sequences with nodes.
__device__ __forceinline__ Item find_item(const TreeArgs& a, uint32_t w) {
  Item it;
  const int H = a.n_kv_heads;
  const uint32_t slot = w >> 3;
  it.rb = (int)(slot % (uint32_t)a.max_nrb);
  int64_t y = (int64_t)(slot / (uint32_t)a.max_nrb) * 8 + (w & 7), base = 0;   // pair, items before the sequence
  it.nrb = 0;
  if (a.wt.n_seq > 0) {
    // branch-free: the table's entries are read at fixed offsets, all at once
    int b = 0, w0 = 0, p0 = 0, t0 = a.wt.tok[0], t1 = a.wt.tok[1], n0 = a.wt.node[0], n1 = a.wt.node[1];
    if (a.wt.n_seq > 1) {
#pragma unroll
      for (int i = 1; i < kKernargSeqs; ++i) {
        const bool here = i < a.wt.n_seq && y >= (int64_t)a.wt.pair[i] * H;
        b = here ? i : b;
        w0 = here ? a.wt.work[i] : w0;
        p0 = here ? a.wt.pair[i] : p0;
        t0 = here ? a.wt.tok[i] : t0;
        t1 = here ? a.wt.tok[i + 1] : t1;
        n0 = here ? a.wt.node[i] : n0;
        n1 = here ? a.wt.node[i + 1] : n1;
      }
    }
    it.b = b;
    base = w0;
    y -= (int64_t)p0 * H;
    it.t0 = t0;
    it.t1 = t1;
    it.n0 = n0;
    it.n = n1 - n0;
  } else {                               // 64 sequences at a time
    const int lane = threadIdx.x & 63;
    for (int b0 = 0;; b0 += 64) {
      if (b0 >= a.batch) return it;
      const int b = b0 + lane;
      int chunks = 0, nrb = 0;
      if (b < a.batch) seq_items(a.cu[b + 1] - a.cu[b], a.cu_nodes[b + 1] - a.cu_nodes[b], a, chunks, nrb);
      const int pairs = nrb > 0 ? chunks + 1 : 0, items = pairs * nrb;
      int pe = pairs, ie = items;
      for (int d = 1; d < 64; d <<= 1) {
        const int po = __shfl_up(pe, d), io = __shfl_up(ie, d);
        if (lane >= d) pe += po, ie += io;
      }
      const unsigned long long in = __ballot(y < (int64_t)pe * H);
      if (in) {
        const int i = __ffsll(in) - 1;
        base += __builtin_amdgcn_readlane(ie - items, i);
        y -= (int64_t)__builtin_amdgcn_readlane(pe - pairs, i) * H;
        it.b = b0 + i;
        break;
      }
      base += __builtin_amdgcn_readlane(ie, 63);
      y -= (int64_t)__builtin_amdgcn_readlane(pe, 63) * H;
    }
    it.t0 = a.cu[it.b];
    it.t1 = a.cu[it.b + 1];
    it.n0 = a.cu_nodes[it.b];
    it.n = a.cu_nodes[it.b + 1] - it.n0;
  }
  seq_items(it.t1 - it.t0, it.n, a, it.chunks, it.nrb);
  it.h = (int)(y % H);
  it.c = (int)(y / H);
  if (it.c > it.chunks || it.rb >= it.nrb) it.nrb = 0;       // past the last pair, or fewer row blocks than the longest
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

// 16 bytes of the query of row r (node r / G, member r % G) from channel c on.
__device__ __forceinline__ u4v q_piece(const TreeArgs& a, const Item& it, int r, int c) {
  return *reinterpret_cast<const u4v*>(a.q + (int64_t)(it.n0 + r / a.group) * a.q_stride + (it.h * a.group + r % a.group) * D + c);
}

// The drafted nodes: a wave takes rows w, w + NW, ... of the block, all at once; a
// lane takes node `lane` for the scores and channels 2 lane, 2 lane + 1 for the
// values.  Nodes a row does not see are skipped, not weighted with zero.  Vector
// products: at 10 us this workgroup ends before those of the chunks (13 us with one
// tile per wave).
template <int NW>
__device__ __forceinline__ void draft_item(const TreeArgs& a, const Item& it, DraftSmem& sm, float* part, int stride) {
  constexpr int PER = R / NW;
  const int wv = threadIdx.x >> 6, lane = threadIdx.x & 63, rows = it.n * a.group;
  const uint16_t* k = a.k_new + (int64_t)(it.n0 + min(lane, it.n - 1)) * a.kv_stride + it.h * D;
  const uint16_t* V = a.v_new + (int64_t)it.n0 * a.kv_stride + it.h * D;
  u4v kw[D / 8];
#pragma unroll
  for (int c = 0; c < D / 8; ++c) kw[c] = *reinterpret_cast<const u4v*>(k + 8 * c);
  for (int i = threadIdx.x; i < it.n * (D / 8); i += 64 * NW)
    *reinterpret_cast<u4v*>(&sm.v[i / (D / 8)][8 * (i % (D / 8))]) =
        *reinterpret_cast<const u4v*>(V + (int64_t)(i / (D / 8)) * a.kv_stride + 8 * (i % (D / 8)));
  for (int i = threadIdx.x; i < R * (D / 8); i += 64 * NW) {
    const int r = i / (D / 8), c = 8 * (i % (D / 8));
    const u4v w = q_piece(a, it, min(it.rb * R + r, rows - 1), c);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint16_t b = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
      sm.q[r][c + j] = a.q_bf16 ? bf16_bits_to_float(b) : half_bits_to_float(b);
    }
  }
  const unsigned long long anc = ancestors(a.parent + it.n0, it.n, lane);
  __syncthreads();
  float s[PER] = {};
#pragma unroll
  for (int c = 0; c < D; c += 4) {
    float kf[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) kf[j] = half_bits_to_float((uint16_t)(kw[c / 8][(c % 8 + j) >> 1] >> (16 * (j & 1))));
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const f4 q = *reinterpret_cast<const f4*>(&sm.q[wv + NW * u][c]);
#pragma unroll
      for (int j = 0; j < 4; ++j) s[u] = __builtin_fmaf(kf[j], q[j], s[u]);
    }
    __builtin_amdgcn_sched_barrier(0);   // else every query piece is read at once, into registers there are none of
  }
#pragma unroll
  for (int u = 0; u < PER; ++u) asm volatile("" : "+v"(s[u]));   // nor are the sums put off until their rows are known to be there
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int row = it.rb * R + wv + NW * u;
    if (row >= rows) continue;
    float* o = part + (int64_t)(wv + NW * u) * stride;
    const unsigned long long see = __shfl(anc, row / a.group);
    const bool mine = (see >> lane) & 1;
    const float sc = mine ? s[u] * a.qscale : -__builtin_inff();
    float m = sc;
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    if (!(m > -__builtin_inff())) m = 0.f;                    // nothing seen, or -inf alone
    const float p = mine ? __builtin_amdgcn_exp2f(sc - m) : 0.f;
    float l = p;
    for (int d = 32; d; d >>= 1) l += __shfl_xor(l, d);
    float o0 = 0.f, o1 = 0.f;
    unsigned long long left = ((unsigned long long)__builtin_amdgcn_readfirstlane((int)(see >> 32)) << 32) |
                              (uint32_t)__builtin_amdgcn_readfirstlane((int)see);
    while (left) {
      const int j = __ffsll(left) - 1;
      left &= left - 1;
      const float pj = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, p), j));
      const uint32_t w = *reinterpret_cast<const uint32_t*>(&sm.v[j][2 * lane]);
      o0 = __builtin_fmaf(pj, half_bits_to_float(w & 0xffff), o0);
      o1 = __builtin_fmaf(pj, half_bits_to_float(w >> 16), o1);
    }
    *reinterpret_cast<float2*>(o + 2 * lane) = make_float2(o0, o1);
    for (int i = lane; i < a.rb; i += 64) o[D + i] = 0.f;
    if (lane == 0) {
      o[D + a.rb] = m;
      o[D + a.rb + 1] = see ? l : -1.f;                       // -1: the node is absent
    }
  }
}

// Two values as fp16 pairs, hi and lo halves, rounded to nearest: on fp16's grid of
// 2^-24 the error then has no direction, and sums of many do not drift.  v - hi is
// exact; the mixed-precision fma takes hi as it is packed (its forms that round to
// fp16 would save one instruction in four and took 3% longer).
__device__ __forceinline__ void pair2(float v0, float v1, uint32_t& hi, uint32_t& lo) {
  hi = __builtin_bit_cast(uint32_t, h2{(_Float16)v0, (_Float16)v1});
  float d0, d1;
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(d0) : "v"(hi), "v"(v0));
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(d1) : "v"(hi), "v"(v1));
  lo = __builtin_bit_cast(uint32_t, h2{(_Float16)d0, (_Float16)d1});
}

// Eight int8 coefficients with their scales in pairs, code * scale = hi + lo exactly:
// the product has 18 bits, hi is it rounded to 11, and the fused multiply-add
// leaves the rest, which lies on the scale's own grid and so in fp16 down to its
// smallest numbers.  A code plus 128 under 0x64 is the fp16 number 1152 + code.  18
// instructions; by way of float32 and pair2 they are 36.
__device__ __forceinline__ void dequant8(u4v w, u4v scale, h8& hi, h8& lo) {
  u4v ph, pl;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t b = __builtin_amdgcn_perm(0x64646464u, w[e >> 1] ^ 0x80808080u, e & 1 ? 0x04030402u : 0x04010400u);
    const uint32_t sw = scale[e];
    const h2 c = __builtin_bit_cast(h2, b) - h2{1152, 1152}, s = __builtin_bit_cast(h2, sw), v = c * s;
    ph[e] = __builtin_bit_cast(uint32_t, v);
    pl[e] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(c, s, -v));
  }
  hi = __builtin_bit_cast(h8, ph);
  lo = __builtin_bit_cast(h8, pl);
}

// Streams of a chunk and KV head; offsets count from the chunk's first 16-token block.
struct Streams {
  rsrc_t k, v, ks, vs;                   // coefficients; int8 block scales
  rsrc_t off, sk, sv;                    // offsets and residual scales from the chunk's first block on
  rsrc_t idx[2], val[2];                 // entries from the chunk's first on
};

// What a wave holds of a tile ahead of its use.
template <int NB, bool C8>
struct Ahead {
  static constexpr int NV = (NB + 1) / 2;
  u4v k[NB], v[NV][2];                   // fp16 coefficients; int8: the first two words
  uint32_t ks[C8 ? NB : 1], vs[C8 ? NB : 1];
  uint32_t oa, ob, oa2, ob2;             // entry ranges of the lane's token, this tile and the next
  uint32_t sk, sv;                       // residual scales
  uint32_t ck, cv, vk, vv;               // entry pair `lane`: channel bytes and code byte, keys and values
};

// Places of a lane in a tile's streams; a tile, a 16-deep step and a block add constants.
struct Lane {
  uint32_t k, v, ks, t2;
};

template <int NB, bool C8>
__device__ __forceinline__ Lane make_lane(int lane) {
  constexpr int rb = 16 * NB;
  const int h = lane >> 5, c = lane & 31, t = row_token(c);
  Lane p;
  if constexpr (C8) {
    p.k = ((t >> 4) * NB * 16 + (t & 15)) * 16 + 8 * h;
    p.v = c * 16 + 8 * h;
  } else {
    p.k = (((t >> 4) * (rb / 8) + h) * 128 + (t & 15) * 8) * 2;
    p.v = (h * rb + c) * 16;
  }
  p.ks = 2 * t;
  p.t2 = 2 * c;
  return p;
}

template <int NB, bool C8>
__device__ __forceinline__ void load_k(Ahead<NB, C8>& f, const Streams& x, const Lane& p, int tile, int T) {
  constexpr int step = TT * 16 * NB * (C8 ? 1 : 2);
#pragma unroll
  for (int s = 0; s < NB; ++s) {
    if constexpr (C8) {
      const u2v w = __builtin_amdgcn_raw_buffer_load_b64(x.k, p.k + 256 * s, tile * step, 0);
      f.k[s].x = w.x;
      f.k[s].y = w.y;
      f.ks[s] = __builtin_amdgcn_raw_buffer_load_b16(x.ks, p.ks, tile * (2 * TT) + s * T * 2, 0);
    } else {
      f.k[s] = __builtin_amdgcn_raw_buffer_load_b128(x.k, p.k + 512 * s, tile * step, 0);
    }
  }
}

// Channels past r_b read whatever follows; their sums are not used.
template <int NB, bool C8>
__device__ __forceinline__ void load_v(Ahead<NB, C8>& f, const Streams& x, const Lane& p, int tile) {
  constexpr int rb = 16 * NB, step = TT * rb * (C8 ? 1 : 2);
#pragma unroll
  for (int k = 0; k < (NB + 1) / 2; ++k) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if constexpr (C8) {
        const u2v w = __builtin_amdgcn_raw_buffer_load_b64(x.v, p.v + 512 * k + u * rb * 16, tile * step, 0);
        f.v[k][u].x = w.x;
        f.v[k][u].y = w.y;
      } else {
        f.v[k][u] = __builtin_amdgcn_raw_buffer_load_b128(x.v, p.v + 512 * k + u * 2 * rb * 16, tile * step, 0);
      }
    }
  }
}

template <int NB, bool C8>
__device__ __forceinline__ void load_vs(Ahead<NB, C8>& f, const Streams& x, const Lane& p, int tile, int T) {
  if constexpr (C8) {
#pragma unroll
    for (int k = 0; k < NB; ++k) f.vs[k] = __builtin_amdgcn_raw_buffer_load_b16(x.vs, p.t2, tile * (2 * TT) + k * T * 2, 0);
  }
}

// Scales and the first 64 entry pairs of a tile whose first entry is e0.
template <int NB, bool C8>
__device__ __forceinline__ void load_entries(Ahead<NB, C8>& f, const Streams& x, const Lane& p, int tile, uint32_t e0, int lane) {
  f.sk = __builtin_amdgcn_raw_buffer_load_b16(x.sk, p.t2, tile * (2 * TT), 0);
  f.sv = __builtin_amdgcn_raw_buffer_load_b16(x.sv, p.t2, tile * (2 * TT), 0);
  f.ck = __builtin_amdgcn_raw_buffer_load_b16(x.idx[0], 2 * lane, e0, 0);
  f.cv = __builtin_amdgcn_raw_buffer_load_b16(x.idx[1], 2 * lane, e0, 0);
  f.vk = __builtin_amdgcn_raw_buffer_load_b8(x.val[0], lane, e0 >> 1, 0);
  f.vv = __builtin_amdgcn_raw_buffer_load_b8(x.val[1], lane, e0 >> 1, 0);
}

template <int NB, bool BF, bool C8>
__global__ __launch_bounds__(64 * kWaves<NB>, kWaves<NB> / 4) void tree_split_kernel(const TreeArgs a) {
  constexpr int NW = kWaves<NB>, NV = (NB + 1) / 2, rb = 16 * NB, stride = D + rb + 4;
  __shared__ TreeSmem<NB, C8> sm;
  const int wv = threadIdx.x >> 6, lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
  const Item it = find_item(a, blockIdx.x);
  if (it.nrb == 0) return;
  const int rows_left = it.n * a.group - it.rb * R;
  float* part = a.part + it.part * R * stride;
  if (it.c == it.chunks) {
    draft_item<NW>(a, it, sm.d, part, stride);
    return;
  }

  // ---- the chunk's streams, and the wave's first tiles in flight -----------------
  const int c0 = it.t0 + it.c * a.split, c1 = it.t1 - c0 > a.split ? c0 + a.split : it.t1, tb = c0 & ~15;
  const int ntile = (c1 - tb + TT - 1) / TT;
  const int64_t T = a.T, T16 = (T + 15) / 16 * 16;
  constexpr int esz = C8 ? 1 : 2;
  const uint32_t* off = a.off + (int64_t)it.h * (T + 1);
  const uint32_t ec0 = off[c0];
  const int64_t eroom = a.res_stride - (int64_t)ec0;   // entries of the slab from the chunk on (ec0 is even)
  const int64_t es = (int64_t)it.h * a.res_stride + (eroom > 0 ? ec0 : 0);
  Streams sx;
  sx.k = make_rsrc(reinterpret_cast<const uint8_t*>(a.coef_k) + ((int64_t)it.h * T16 + tb) * rb * esz, (T16 - tb) * rb * esz);
  sx.v = make_rsrc(reinterpret_cast<const uint8_t*>(a.coef_v) + ((int64_t)it.h * T16 + tb) * rb * esz, (T16 - tb) * rb * esz);
  sx.off = make_rsrc(off + tb, (T + 1 - tb) * 4);
  sx.sk = make_rsrc(a.scale_k + (int64_t)it.h * T + tb, (T - tb) * 2);
  sx.sv = make_rsrc(a.scale_v + (int64_t)it.h * T + tb, (T - tb) * 2);
  sx.idx[0] = make_rsrc(a.idx_k + es, eroom);
  sx.idx[1] = make_rsrc(a.idx_v + es, eroom);
  sx.val[0] = make_rsrc(a.val_k + es / 2, eroom / 2);
  sx.val[1] = make_rsrc(a.val_v + es / 2, eroom / 2);
  if constexpr (C8) {
    sx.ks = make_rsrc(a.cscale_k + (int64_t)it.h * NB * T + tb, (NB * T - tb) * 2);
    sx.vs = make_rsrc(a.cscale_v + (int64_t)it.h * NB * T + tb, (NB * T - tb) * 2);
  }
  const int Ti = (int)T;
  const int wvu = __builtin_amdgcn_readfirstlane(wv);
  const int last = ntile - 1, j0 = min(wvu, last);      // tiles past the last are read as the last and not used
  const auto load_off = [&](int j, uint32_t& oa, uint32_t& ob) {
    const int t = j * TT + (lane & 31);                // tokens outside the chunk hold no entries
    oa = __builtin_amdgcn_raw_buffer_load_b32(sx.off, (uint32_t)min(max(t, c0 - tb), c1 - tb) * 4, 0, 0) - ec0;
    ob = __builtin_amdgcn_raw_buffer_load_b32(sx.off, (uint32_t)min(max(t + 1, c0 - tb), c1 - tb) * 4, 0, 0) - ec0;
  };
  const Lane lp = make_lane<NB, C8>(lane);
  Ahead<NB, C8> f;
  load_off(j0, f.oa, f.ob);
  load_off(min(j0 + NW, last), f.oa2, f.ob2);
  load_k<NB, C8>(f, sx, lp, j0, Ti);

  // ---- query fragments, and q~ = B^K q as fp16 pairs (16x16x4 float32 products) ---
  constexpr int TILES = 2 * NB, PER = (TILES + NW - 1) / NW;
  const int g = lane >> 4, c16 = lane & 15;
  const uint16_t* bk = a.basis + (int64_t)it.b * a.basis_b_stride + (int64_t)(it.h * 2) * rb * D;
  u4v bw[PER][4];
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int tile = wv + NW * u;
#pragma unroll
    for (int s = 0; s < 4; ++s)
      if (tile < TILES) bw[u][s] = *reinterpret_cast<const u4v*>(bk + (16 * (tile / 2) + c16) * D + 32 * s + 8 * g);
  }
  for (int i = threadIdx.x; i < 8 * 64; i += 64 * NW) {
    const int ln = i & 63, s = i >> 6, r = ln & 31;
    u4v w = {0, 0, 0, 0};
    // a query meets its own column of every product alone: an absent node's may be anything
    if (r < rows_left) w = q_piece(a, it, it.rb * R + r, 16 * s + 8 * (ln >> 5));
    sm.qf[s][ln] = w;
  }
  if (threadIdx.x < R) sm.big[threadIdx.x] = 0.f;
  if (threadIdx.x < D) sm.odd[threadIdx.x] = 0;
  WaveTile& w = sm.w[wv];
  for (int i = lane; i < (int)((sizeof(w.k) + sizeof(w.v)) / 16); i += 64) reinterpret_cast<u4v*>(&w)[i] = u4v{0, 0, 0, 0};
  __syncthreads();
  {
    f4 q[PER];
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int tile = wv + NW * u, n = tile % 2;
      float big = 0.f;
      f4 c = {0.f, 0.f, 0.f, 0.f};
      if (tile < TILES) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const u4v qw = sm.qf[2 * s + (g >> 1)][32 * (g & 1) + 16 * n + c16];   // channels 32 s + 8 g + j
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint16_t qb = (uint16_t)(qw[j >> 1] >> (16 * (j & 1))), bb = (uint16_t)(bw[u][s][j >> 1] >> (16 * (j & 1)));
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
      big = fmaxf(big, __shfl_xor(big, 16));
      big = fmaxf(big, __shfl_xor(big, 32));
      if (tile < TILES && g == 0) atomicMax(reinterpret_cast<int*>(&sm.big[16 * n + c16]), __builtin_bit_cast(int, big));
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int tile = wv + NW * u;
      if (tile >= TILES) continue;
      const float dn = __builtin_ldexpf(1.f, -row_down(sm.big[16 * (tile % 2) + c16]));
      h4 hi, lo;                                       // basis rows 16 (tile / 2) + 4 g + i, row 16 (tile % 2) + c16
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float v = q[u][i] * dn;
        hi[i] = (_Float16)v;
        lo[i] = (_Float16)(v - (float)hi[i]);
      }
      const int ln = 32 * (g >> 1) + 16 * (tile % 2) + c16;
      reinterpret_cast<h4*>(&sm.qt[0][tile / 2][ln])[g & 1] = hi;
      reinterpret_cast<h4*>(&sm.qt[1][tile / 2][ln])[g & 1] = lo;
    }
  }
  const bool scaled = __ballot(row_down(sm.big[col]) != 0) != 0;
  uint32_t e0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)f.oa);
  load_entries<NB, C8>(f, sx, lp, j0, e0, lane);
  load_vs<NB, C8>(f, sx, lp, j0, Ti);
  load_v<NB, C8>(f, sx, lp, j0);
  __syncthreads();                       // q~ is whole

  f16v acc_a[NV], acc_r[D / 32];         // a~ and the residual channels: (channel 8 a + 4 h + i of the block, row col)
  float m = 0.f, l = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) acc_a[k] = f16v{};
#pragma unroll
  for (int k = 0; k < D / 32; ++k) acc_r[k] = f16v{};
  const float inf = __builtin_inff();
  float lim = -inf;                      // a score past it moves the row's reference; -inf: the row has none yet
  // acc_r is the residual sum times rs, a power of two of the row's own: 2^-ex, or more
  // where the row's largest weight p |s^V| so far (in sm.m) would not reach 1/4 with it
  int ex = kNoScale;                     // |s^V| < 2^ex of the tiles so far
  float exf = __builtin_ldexpf(1.f, kNoScale), rs = __builtin_ldexpf(1.f, kMost);
  sm.m[wv][col] = 0.f;
  const auto unit_of = [&](float top) { return top > 0.f ? min(max(-ex, -1 - __builtin_amdgcn_frexp_expf(top)), kMost) : kMost; };

#pragma unroll 1
  for (int j = wvu; j < ntile; j += NW) {
    const int t0 = tb + j * TT, jn = min(j + NW, last);
    const bool edge = t0 < c0 || t0 + TT > c1;
    // Loads return in order, and a wait for one is a wait for those before it.  A
    // tile's key coefficients, entries and value coefficients are requested
    // in that order, each once its predecessor's registers are free.
    // ---- basis part of the scores: register 8 u + e is token 16 u + 8 h + e, row col
    f16v sb = {}, sr = {};
#pragma unroll
    for (int s = 0; s < NB; ++s) {
      const h8 qh = __builtin_bit_cast(h8, sm.qt[0][s][lane]), ql = __builtin_bit_cast(h8, sm.qt[1][s][lane]);
      if constexpr (C8) {
        const uint32_t sc = (f.ks[s] & 0xffff) * 0x10001u;
        h8 kh, kl;
        dequant8(f.k[s], u4v{sc, sc, sc, sc}, kh, kl);
        sb = mfma_h(kh, qh, sb);
        sb = mfma_h(kh, ql, sb);
        sb = mfma_h(kl, qh, sb);
      } else {
        sb = mfma_h(__builtin_bit_cast(h8, f.k[s]), qh, sb);
        sb = mfma_h(__builtin_bit_cast(h8, f.k[s]), ql, sb);
      }
    }
    load_k<NB, C8>(f, sx, lp, jn, Ti);
    // ---- entries of the next tile and offsets of the one after
    const uint32_t oa = f.oa, ob = f.ob, sk = f.sk, sv = f.sv, ck = f.ck, cv = f.cv, vk = f.vk, vv = f.vv;
    const uint32_t en = e0;
    f.oa = f.oa2;
    f.ob = f.ob2;
    e0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)f.oa);
    if constexpr (C8) {
      if (lane < 32) {
#pragma unroll
        for (int k = 0; k < NB; ++k) sm.vs[wv][k][lane] = (uint16_t)f.vs[k];
      }
    }
    load_off(min(jn + NW, last), f.oa2, f.ob2);
    load_entries<NB, C8>(f, sx, lp, jn, e0, lane);
    load_vs<NB, C8>(f, sx, lp, jn, Ti);

    // ---- scales, one lane per token
    const bool own = ob > oa;
    const float fk = own ? half_bits_to_float((uint16_t)sk) : 0.f, fv = own ? half_bits_to_float((uint16_t)sv) : 0.f;
    const bool odd_k = !(fabsf(fk) < inf), odd_v = !(fabsf(fv) < inf);
    if (__ballot(!odd_v && fabsf(fv) > exf)) {           // rare: larger value scales
      int e = !odd_v && fv != 0.f ? __builtin_amdgcn_frexp_expf(fv) : kNoScale;
      for (int d = 32; d; d >>= 1) e = max(e, __shfl_xor(e, d));
      ex = e;
      exf = __builtin_ldexpf(1.f, e);
      const int er = unit_of(sm.m[wv][col]);
      const float g = __builtin_ldexpf(1.f, er + 1 - __builtin_amdgcn_frexp_expf(rs));
      rs *= g;
#pragma unroll
      for (int k = 0; k < D / 32; ++k) acc_r[k] *= g;
      if (lim > -inf) lim = fminf(kHead, kFull - (ex + er));
    }
    const bool odd = __ballot(odd_k || odd_v) != 0;
    // A key scale that is not finite goes with its entries into the code tile.  A
    // value scale that is not: every row sees its token, so its entries'
    // channels end as infinities of their sign or NaN whatever the rest is; they
    // are noted, and left out here.
    w.sk[lane & 31] = odd_k ? a.qscale : fk * a.qscale;
    w.sv[lane & 31] = odd_v ? 0.f : fv;
    // ---- entries into the code tiles, 64 pairs at a time (ranks are even, so a pair belongs to one token)
    const uint32_t e1 = (uint32_t)__builtin_amdgcn_readlane((int)ob, 31);
    const uint32_t np = e1 > en ? min(e1 - en, (uint32_t)(TT * D)) / 2 : 0u;
    uint32_t at_k, at_v;                               // places of the first batch
    const auto scatter = [&](uint32_t b0, int carry, uint32_t pk, uint32_t pv, uint32_t qk, uint32_t qv, uint32_t& ak, uint32_t& av) {
      w.mark[lane] = 0;
      wave_lds_sync();
      const uint32_t at = (oa - en) / 2 - b0;
      w.mark[lane < 32 && own && at < 64 ? at : 64 + lane] = (uint8_t)(lane + 1);
      wave_lds_sync();
      const int tok = max(incl_max((int)w.mark[lane]), carry);
      const bool live = b0 + lane < np && tok > 0;
      const int t = (tok - 1) & (TT - 1), kr = key_row(t) * kKRow;
      const uint32_t k0 = live ? kr + (pk & (D - 1)) : kNoKey, k1 = live ? kr + ((pk >> 8) & (D - 1)) : kNoKey;
      const uint32_t v0 = live ? value_place(pv & (D - 1), t) : kNoValue, v1 = live ? value_place((pv >> 8) & (D - 1), t) : kNoValue;
      ak = k0 | k1 << 16;
      av = v0 | v1 << 16;
      const float a0 = (float)int4_value(qk), a1 = (float)int4_value(qk >> 4), b0f = (float)int4_value(qv), b1f = (float)int4_value(qv >> 4);
      uint16_t wk0 = code_bits<BF>(a0), wk1 = code_bits<BF>(a1), wv0 = h_bits(b0f), wv1 = h_bits(b1f);
      if (odd) {
        const uint32_t t2 = (uint32_t)(j * TT + t) * 2;
        const float tk = half_bits_to_float(__builtin_amdgcn_raw_buffer_load_b16(sx.sk, t2, 0, 0));
        const float tv = half_bits_to_float(__builtin_amdgcn_raw_buffer_load_b16(sx.sv, t2, 0, 0));
        __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
        if (!(fabsf(tk) < inf)) wk0 = code_bits<BF>(a0 * tk), wk1 = code_bits<BF>(a1 * tk);
        if (!(fabsf(tv) < inf) && live) {
          const float x0 = b0f * tv, x1 = b1f * tv;
          atomicOr(&sm.odd[pv & (D - 1)], x0 > 0.f ? 1u : x0 < 0.f ? 2u : 4u);
          atomicOr(&sm.odd[(pv >> 8) & (D - 1)], x1 > 0.f ? 1u : x1 < 0.f ? 2u : 4u);
        }
      }
      w.k[k0] = wk0;
      w.k[k1] = wk1;
      w.v[v0] = wv0;
      w.v[v1] = wv1;
      return __builtin_amdgcn_readlane(tok, 63);
    };
    int carry = scatter(0, 0, ck, cv, vk, vv, at_k, at_v);
#pragma unroll 1
    for (uint32_t b0 = 64; b0 < np; b0 += 64) {        // more than 128 entries: read as they come
      const uint32_t e = en + 2 * (b0 + lane);
      uint32_t x0, x1;
      carry = scatter(b0, carry, __builtin_amdgcn_raw_buffer_load_b16(sx.idx[0], e, 0, 0), __builtin_amdgcn_raw_buffer_load_b16(sx.idx[1], e, 0, 0),
                      __builtin_amdgcn_raw_buffer_load_b8(sx.val[0], e >> 1, 0, 0), __builtin_amdgcn_raw_buffer_load_b8(sx.val[1], e >> 1, 0, 0), x0, x1);
      // nothing of this rare path may look pending after it: the compiler would
      // have every tile wait for all its loads
      __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
    }
    wave_lds_sync();

    // ---- residual part of the scores
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const u4v kc = *reinterpret_cast<const u4v*>(&w.k[col * kKRow + 16 * s + 8 * h]);
      sr = mfma_q<BF>(kc, sm.qf[s][lane], sr);
    }
    if (scaled) {                        // all but zero queries; the branch keeps what follows out of the products' registers
      const float up = __builtin_ldexpf(1.f, row_down(sm.big[col]));
#pragma unroll
      for (int i = 0; i < 16; ++i) sb[i] = __builtin_fmaf(sb[i], up, -m);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) sb[i] -= m;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const f4 ks = *reinterpret_cast<const f4*>(&w.sk[16 * u + 8 * h + 4 * q]);
#pragma unroll
        for (int i = 0; i < 4; ++i) sb[8 * u + 4 * q + i] = __builtin_fmaf(ks[i], sr[8 * u + 4 * q + i], sb[8 * u + 4 * q + i]);
      }
    }
    if (edge) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int t = t0 + 16 * u + 8 * h + e;
          if (t < c0 || t >= c1) {
            sb[8 * u + e] = -inf;
            if constexpr (!C8) {         // tokens outside the chunk may hold anything
#pragma unroll
              for (int k = 0; k < NV; ++k) {
                h8 av = __builtin_bit_cast(h8, f.v[k][u]);
                av[e] = (_Float16)0.f;
                f.v[k][u] = __builtin_bit_cast(u4v, av);
              }
            }
          }
        }
      }
    }
    // ---- a row's reference moves for its first score above -inf, and when one exceeds it
    // by far; the scale of its residual weights follows, also where a score allows a
    // weight that would exceed fp16's range
    float mx = sb[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sb[i]);
    if (__ballot(mx > lim)) {
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const bool past = mx > lim;
      float by = past && (lim == -inf || mx > kHead) ? mx - kUp : 0.f;
      by = mx - by > kHead ? mx : by;    // scores of 2^27 and more come in steps beyond kUp
      const float fall = lim > -inf ? __builtin_amdgcn_exp2f(-by) : 1.f;
      m += by;
      l *= fall;
#pragma unroll
      for (int i = 0; i < 16; ++i) sb[i] -= by;
      float top = 0.f;
      int at = 8 * h;
      asm("" : "+v"(at));                // what follows is computed here and again below: kept, it has no registers
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f4 s = *reinterpret_cast<const f4*>(&w.sv[at + 16 * (q >> 1) + 4 * (q & 1)]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = sb[4 * q + i];
          asm("" : "+v"(x));
          top = fmaxf(top, __builtin_amdgcn_exp2f(x) * fabsf(s[i]));
        }
      }
      top = fmaxf(fmaxf(top, __shfl_xor(top, 32)), sm.m[wv][col] * fall);
      const int was = __builtin_amdgcn_frexp_expf(rs) - 1, er = past ? unit_of(top) : was;
      const float g = __builtin_ldexpf(fall, er - was);
      if (__ballot(fall != 1.f)) {
#pragma unroll
        for (int k = 0; k < NV; ++k) acc_a[k] *= fall;
      }
      if (__ballot(g != 1.f) && j > wvu) {     // nothing is summed up yet at the wave's first tile
#pragma unroll
        for (int k = 0; k < D / 32; ++k) acc_r[k] *= g;
      }
      if (past) {
        rs = __builtin_ldexpf(1.f, er);
        lim = fminf(kHead, kFull - (ex + er));
        sm.m[wv][col] = top;
      }
    }
    // ---- probabilities as fp16 pairs, plain and times the value scales; values:
    // channel blocks of the basis, then of the residual
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const f4 s0 = *reinterpret_cast<const f4*>(&w.sv[16 * u + 8 * h]), s1 = *reinterpret_cast<const f4*>(&w.sv[16 * u + 8 * h + 4]);
      u4v ph, pl, rh, rl;
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float v0 = __builtin_amdgcn_exp2f(sb[8 * u + e]), v1 = __builtin_amdgcn_exp2f(sb[8 * u + e + 1]);
        const float x0 = (e < 4 ? s0[e & 3] : s1[e & 3]) * rs, x1 = (e < 4 ? s0[(e & 3) + 1] : s1[(e & 3) + 1]) * rs;
        sum[0] += v0;
        sum[1] += v1;
        uint32_t hi, lo;
        pair2(v0, v1, hi, lo);
        ph[e >> 1] = hi;
        pl[e >> 1] = lo;
        pair2(v0 * x0, v1 * x1, hi, lo);
        rh[e >> 1] = hi;
        rl[e >> 1] = lo;
      }
      l += sum[0] + sum[1];
      const h8 p0 = __builtin_bit_cast(h8, ph), p1 = __builtin_bit_cast(h8, pl), r0 = __builtin_bit_cast(h8, rh), r1 = __builtin_bit_cast(h8, rl);
#pragma unroll
      for (int k = 0; k < D / 32; ++k) {
        const h8 vc = __builtin_bit_cast(h8, *reinterpret_cast<const u4v*>(&w.v[value_place(32 * k + col, 16 * u + 8 * h)]));
        acc_r[k] = mfma_h(vc, r0, acc_r[k]);
        acc_r[k] = mfma_h(vc, r1, acc_r[k]);
      }
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        if constexpr (C8) {
          const u4v sw = *reinterpret_cast<const u4v*>(&sm.vs[wv][min(2 * k + (col >> 4), NB - 1)][16 * u + 8 * h]);
          h8 hi, lo;
          dequant8(f.v[k][u], sw, hi, lo);
          if (edge) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (t0 + 16 * u + 8 * h + e < c0 || t0 + 16 * u + 8 * h + e >= c1) hi[e] = lo[e] = (_Float16)0.f;
          }
          acc_a[k] = mfma_h(hi, p0, acc_a[k]);
          acc_a[k] = mfma_h(hi, p1, acc_a[k]);
          acc_a[k] = mfma_h(lo, p0, acc_a[k]);
        } else {
          acc_a[k] = mfma_h(__builtin_bit_cast(h8, f.v[k][u]), p0, acc_a[k]);
          acc_a[k] = mfma_h(__builtin_bit_cast(h8, f.v[k][u]), p1, acc_a[k]);
        }
      }
    }
    load_v<NB, C8>(f, sx, lp, jn);
    // ---- the code tiles go back to zero
    wave_lds_sync();
    if (np > 64) {
      for (int i = lane; i < (int)((sizeof(w.k) + sizeof(w.v)) / 16); i += 64) reinterpret_cast<u4v*>(&w)[i] = u4v{0, 0, 0, 0};
    } else {
      w.k[at_k & 0xffff] = 0;
      w.k[at_k >> 16] = 0;
      w.v[at_v & 0xffff] = 0;
      w.v[at_v >> 16] = 0;
    }
    wave_lds_sync();
  }

  // ---- join the waves: common reference per row, then sums in wave order -----------
  l += __shfl_xor(l, 32);
  const bool none = lim == -inf && l == 0.f;   // no score above -inf, nor one that is no number
  if (h == 0) {
    sm.m[wv][col] = none ? -inf : m;
    sm.l[wv][col] = l;
  }
  __syncthreads();                       // the code tiles are done with
  float ms = -inf;
#pragma unroll
  for (int u = 0; u < NW; ++u) ms = fmaxf(ms, sm.m[u][col]);
  const float mine = none ? 0.f : __builtin_amdgcn_exp2f(m - ms), unit = __builtin_ldexpf(1.f, 1 - __builtin_amdgcn_frexp_expf(rs));
#pragma unroll
  for (int k = 0; k < D / 32; ++k)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<f4*>(&sm.acc[wv][col][32 * k + 8 * q + 4 * h]) =
          f4{acc_r[k][4 * q], acc_r[k][4 * q + 1], acc_r[k][4 * q + 2], acc_r[k][4 * q + 3]} * (mine * unit);
  __syncthreads();
  for (int i = threadIdx.x; i < R * (D / 4); i += 64 * NW) {
    const int r = i / (D / 4), c = 4 * (i % (D / 4));
    f4 s = {0, 0, 0, 0};
#pragma unroll
    for (int u = 0; u < NW; ++u) s += *reinterpret_cast<const f4*>(&sm.acc[u][r][c]);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (const uint32_t o = sm.odd[c + k]) s[k] = o == 1 ? inf : o == 2 ? -inf : __builtin_nanf("");
    if (r < rows_left) *reinterpret_cast<f4*>(part + r * stride + c) = s;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (32 * k + 8 * q < rb)
        *reinterpret_cast<f4*>(&sm.acc[wv][col][32 * k + 8 * q + 4 * h]) =
            f4{acc_a[k][4 * q], acc_a[k][4 * q + 1], acc_a[k][4 * q + 2], acc_a[k][4 * q + 3]} * mine;
  __syncthreads();
  for (int i = threadIdx.x; i < R * (rb / 4); i += 64 * NW) {
    const int r = i / (rb / 4), c = 4 * (i % (rb / 4));
    f4 s = {0, 0, 0, 0};
#pragma unroll
    for (int u = 0; u < NW; ++u) s += *reinterpret_cast<const f4*>(&sm.acc[u][r][c]);
    if (r < rows_left) *reinterpret_cast<f4*>(part + r * stride + D + c) = s;
  }
  if (threadIdx.x < R && (int)threadIdx.x < rows_left) {
    const int r = threadIdx.x;
    float ms = -inf, ls = 0.f;
#pragma unroll
    for (int u = 0; u < NW; ++u) ms = fmaxf(ms, sm.m[u][r]);
#pragma unroll
    for (int u = 0; u < NW; ++u)
      if (sm.m[u][r] > -inf) ls += sm.l[u][r] * __builtin_amdgcn_exp2f(sm.m[u][r] - ms);
    part[r * stride + D + rb] = ms;
    part[r * stride + D + rb + 1] = ls;
  }
}

template <int NB, bool BF>
void launch_tree_b(const TreeArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.n_pairs + 7) / 8 * 8 * a.max_nrb)), block(64 * kWaves<NB>);
  if (a.c8) hipLaunchKernelGGL((tree_split_kernel<NB, BF, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((tree_split_kernel<NB, BF, false>), grid, block, 0, s, a);
}

template <bool BF>
void launch_tree_split(const TreeArgs& a, hipStream_t s) {
  switch (a.rb / 16) {
    case 1: launch_tree_b<1, BF>(a, s); break;
    case 2: launch_tree_b<2, BF>(a, s); break;
    case 3: launch_tree_b<3, BF>(a, s); break;
    case 4: launch_tree_b<4, BF>(a, s); break;
    case 5: launch_tree_b<5, BF>(a, s); break;
    case 6: launch_tree_b<6, BF>(a, s); break;
    case 7: launch_tree_b<7, BF>(a, s); break;
    default: launch_tree_b<8, BF>(a, s); break;
  }
}

}  // namespace
}  // namespace dwkv
