// Attention of one new token per sequence over a paged dense cache, gfx950.
//
//   out[b][hq] = sum_t p_t v_t,  p = softmax_t(sm_scale q . k_t)
// over the tokens t of the last `window` (or all) that sequence b holds in pages.
// Bound by HBM: 4 d bytes per token and KV head against 4 G d flop, so the products
// run on 16x16x32 matrix instructions whatever the group is and everything else is
// about keeping loads in flight.
//  * Lengths and page tables are device data (a captured graph follows them), so
//    the work is shared out on the device: tiles of 32 tokens of every (sequence,
//    KV head, block of 16 heads) in one list, an equal run of it for each wave.  Where
//    one workgroup can read a pair's tokens in the time that the second launch takes, each
//    pair has one, and the longest sequences come first.
//  * Keys lie in tiles of 16 tokens x 8 channels and values in blocks of 8 tokens, as
//    the factorized cache's coefficients do: each wave load covers whole 128-byte lines
//    and is an operand as it stands.  Scores come out with a lane's head down its
//    column (tokens 4g + i of either 16); two lane-group swaps turn the probabilities
//    into the second product's operand (tokens 8g + j).
//  * Probabilities: the reference leaves a row's largest at 2^9 and moves when one
//    passes 2^15.5, as 2^9 leaves small ones room in fp16's range.  They enter the
//    product as two fp16 or three bf16 terms (22 and 24 bits): the values' type has 11
//    or 8, which would be the output's error.  Only what is finite can be multiplied like
//    that: where a sum is not, its infinities are added up by themselves.
//  * A wave writes what it has of a pair that it shares with others as a partial, and
//    a pair of its own as output; the waves of a workgroup that all work on one
//    pair join in LDS first.  page_merge_kernel joins the partials.
#include <algorithm>

#include "internal.h"

namespace dwkv {
namespace {

constexpr int kPT = 64 * kPageWaves;
constexpr int kSingleTiles = 128, kSingleBits = 8;    // most tiles of a pair that one workgroup takes, and their bits
constexpr int kRanked = 256;             // sequences that are taken longest first
constexpr float kFar = 0x1.fffffep127f;
constexpr float kNoRef = -kFar;          // reference of a row without scores: below every other number
constexpr float kRefTop = 9.f, kRefMove = 15.5f;

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 brain8 __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef uint32_t uint4_t __attribute__((ext_vector_type(4)));

template <int TY>
__device__ __forceinline__ float4_t product(uint4_t a, uint4_t b, float4_t c) {
  if constexpr (TY == DWKV_F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(brain8, a), __builtin_bit_cast(brain8, b), c, 0, 0, 0);
}

// Two floats rounded to the type and packed; what is left of them.
template <int TY>
__device__ __forceinline__ uint32_t take(float& a, float& b) {
  if constexpr (TY == DWKV_F16) {
    typedef _Float16 pair __attribute__((ext_vector_type(2)));
    const pair p = {(_Float16)a, (_Float16)b};
    a -= (float)p[0];
    b -= (float)p[1];
    return __builtin_bit_cast(uint32_t, p);
  } else {
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    const pair p = {(__bf16)a, (__bf16)b};
    a -= (float)p[0];
    b -= (float)p[1];
    return __builtin_bit_cast(uint32_t, p);
  }
}

// The halves of a pair that are infinite or NaN; 0 for others.
template <int TY>
__device__ __forceinline__ uint32_t not_finite(uint32_t v) {
  constexpr uint32_t lo = TY == DWKV_F16 ? 0x7c00u : 0x7f80u, hi = lo << 16;
  return ((v & lo) == lo ? v & 0xffffu : 0u) | ((v & hi) == hi ? v & 0xffff0000u : 0u);
}

// sum + x f of a partial's x and its weight f, which is 0 below float32's range: an infinite x counts all the same.
__device__ __forceinline__ float plus(float sum, float x, float f) { return f != 0.f ? __builtin_fmaf(x, f, sum) : x - x == 0.f ? sum : sum + x; }

struct Span {               // tokens of a sequence that its new one attends to
  int start, len;
};
__device__ __forceinline__ Span span_of(const PageArgs& a, int b) {
  const int64_t room = (int64_t)a.max_pages << (a.page_shift + 4);
  Span s;
  s.len = (int)min((int64_t)max(a.len[b], 0), room);
  s.start = a.window > 0 ? max(0, s.len - a.window) : 0;
  return s;
}
__device__ __forceinline__ int tiles_of(Span s) { return (s.len + kPageTile - 1) / kPageTile - s.start / kPageTile; }

// How the list of `total` tiles is shared out: runs of `wg` for each workgroup and of `per` for
// each of its waves.  Lists of less than a tile a wave go to all workgroups evenly, as
// what one compute unit can read at a time is the limit there.
struct Share {
  int wg, per;
};
__device__ __forceinline__ Share share_of(int total) {
  Share s;
  s.per = max(1, (total + kPageWG * kPageWaves - 1) / (kPageWG * kPageWaves));
  s.wg = s.per > 1 ? s.per * kPageWaves : max(1, (total + kPageWG - 1) / kPageWG);
  return s;
}

// Slot of the partial that run [x, ...) of wave w writes for the pair that begins at p0.
__device__ __forceinline__ int slot_of(int w, int x, int p0) { return 2 * w + (x > p0 ? 0 : 1); }

// The sequence with `rank` ones before it in the order from the longest to the shortest, equal ones as
// they come: up to kRanked sequences, up to 2^kSingleBits - 1 tiles.  A bit at a time: those with it
// come before those without.
__device__ __forceinline__ int of_rank(const PageArgs& a, int rank, int lane) {
  constexpr int N = kRanked / 64;
  int t[N];
  unsigned long long left[N];            // those that share the bits so far
#pragma unroll
  for (int c = 0; c < N; ++c) {
    const int i = 64 * c + lane;
    t[c] = 0;
    left[c] = 0;
    if (64 * c < a.batch) {
      left[c] = __ballot(i < a.batch);
      if (i < a.batch) t[c] = tiles_of(span_of(a, i));
    }
  }
#pragma unroll
  for (int bit = kSingleBits - 1; bit >= 0; --bit) {
    unsigned long long set[N];
    int n = 0;
#pragma unroll
    for (int c = 0; c < N; ++c) {
      set[c] = 0;
      if (64 * c < a.batch) set[c] = __ballot((t[c] >> bit) & 1) & left[c];
      n += (int)__popcll(set[c]);
    }
    const bool in = rank < n;
    if (!in) rank -= n;
#pragma unroll
    for (int c = 0; c < N; ++c) left[c] = in ? set[c] : left[c] & ~set[c];
  }
  int b = 0;
#pragma unroll
  for (int c = 0; c < N; ++c) {
    const int n = (int)__popcll(left[c]);
    const int below = __builtin_amdgcn_mbcnt_hi((uint32_t)(left[c] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)left[c], 0));
    const unsigned long long it = __ballot((left[c] >> lane & 1) && below == rank);
    if (it) b = 64 * c + (int)__builtin_ctzll(it);
    rank = rank < n ? -1 : rank - n;
  }
  return __builtin_amdgcn_readfirstlane(b);
}

// SINGLE: grid (KV heads x blocks of 16 heads, B), a workgroup for each pair, the output
// written at once.  Else kPageWG workgroups, and a merge after it.
template <int D, int TY, bool SINGLE>
__global__ __launch_bounds__(kPT) void page_split_kernel(const PageArgs a) {
  constexpr int KS = D / 32, VB = D / 16, PS = D + 4;
  extern __shared__ __align__(16) float smem[];
  __shared__ int sums[kPageWaves];
  float* joined = smem;                                        // [waves][rows][PS]
  int* pre = reinterpret_cast<int*>(smem + kPageWaves * a.rows * PS);   // [B+1] tiles before each sequence
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 15, g = lane >> 4, pairs = a.n_kv_heads * a.n_rb;
  const int w = blockIdx.x * kPageWaves + wv;
  const bool few = a.batch <= 64;                              // a lane for each sequence
  int inc = 0;                                                 // with few: tiles up to this lane's sequence
  int wg0, wg1, x, end, b, wgp, wgp0, wgT;
  bool join;
  int early = -1;                                              // SINGLE: ids of the wave's first pages, before the length is known
  const auto before = [&](int i) {
    return __builtin_amdgcn_readfirstlane(few ? (i ? __builtin_amdgcn_readlane(inc, i - 1) : 0) : pre[i]);
  };
  // the sequence that holds list position i: the first with tiles up to its end * pairs > i
  const auto seq_at = [&](int i) {
    if (few) return __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(__ballot(lane < a.batch && inc * pairs > i)));
    int lo = 0, hi = a.batch - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (pre[mid + 1] * pairs > i) hi = mid; else lo = mid + 1;
    }
    return __builtin_amdgcn_readfirstlane(lo);
  };
  if constexpr (SINGLE) {
    b = blockIdx.y;
    if (a.longest_first) {               // the order in which workgroups start: short ones fill the end
      b = of_rank(a, blockIdx.y, lane);
    }
    wgp = blockIdx.x;
    const int p = ((wv * kPageTile) >> (a.page_shift + 4)) + lane;
    if (p < a.max_pages) early = a.table[(int64_t)b * a.max_pages + p];
    wgT = __builtin_amdgcn_readfirstlane(tiles_of(span_of(a, b)));
    wg0 = wgp0 = x = 0;
    wg1 = end = wgT;
    join = true;
  } else {
    int total = 0;
    if (few) {
      inc = lane < a.batch ? tiles_of(span_of(a, lane)) : 0;
      for (int d = 1; d < a.batch; d <<= 1) {
        const int o = __shfl_up(inc, d);
        if (lane >= d) inc += o;
      }
      total = __builtin_amdgcn_readlane(inc, a.batch - 1);
      if (blockIdx.x == 0 && wv == 0) {
        if (lane < a.batch) a.plan[lane + 1] = inc;
        if (lane == 0) a.plan[0] = 0;
      }
    } else {
      for (int b0 = 0; b0 < a.batch; b0 += kPT) {
        const int i = b0 + (int)threadIdx.x;
        int sum = i < a.batch ? tiles_of(span_of(a, i)) : 0;
        for (int d = 1; d < 64; d <<= 1) {
          const int o = __shfl_up(sum, d);
          if (lane >= d) sum += o;
        }
        if (lane == 63) sums[wv] = sum;
        __syncthreads();
        int first = total;
        for (int k = 0; k < kPageWaves; ++k) {
          if (k < wv) first += sums[k];
          total += sums[k];
        }
        if (i < a.batch) {
          pre[i + 1] = first + sum;
          if (blockIdx.x == 0) a.plan[i + 1] = first + sum;
        }
        __syncthreads();
      }
      if (threadIdx.x == 0) {
        pre[0] = 0;
        if (blockIdx.x == 0) a.plan[0] = 0;
      }
      __syncthreads();
    }
    total *= pairs;
    const Share s = share_of(total);
    wg0 = min(total, (int)blockIdx.x * s.wg);
    wg1 = min(total, wg0 + s.wg);
    if (wg0 >= wg1) return;
    x = min(wg1, wg0 + wv * s.per);
    end = min(wg1, x + s.per);
    b = seq_at(wg0);
    wgT = before(b + 1) - before(b);
    wgp = (wg0 - before(b) * pairs) / wgT;
    wgp0 = before(b) * pairs + wgp * wgT;
    join = wg1 <= wgp0 + wgT;                                  // one pair for the whole workgroup
  }

  float ref = kNoRef, l = 0.f;
  float4_t o[VB];
#pragma unroll
  for (int i = 0; i < VB; ++i) o[i] = 0.f;

  // the waves of a workgroup with one pair take its tiles in turn, so that it reads on in one place
  const int turn = join ? kPageWaves : 1;
  const int stop = join ? wg1 : end;
  if (join) x = wg0 + wv;
  if (!join && x < end) b = seq_at(x);
  while (x < stop) {
    int pair = wgp, p0 = wgp0, T = wgT;
    if (!join) {
      const int pb = before(b);
      T = before(b + 1) - pb;
      if (T == 0 || x >= (pb + T) * pairs) {
        ++b;
        continue;
      }
      pair = (x - pb * pairs) / T;
      p0 = pb * pairs + pair * T;
    }
    const int n = (min(stop, p0 + T) - x + turn - 1) / turn;
    const int h = pair / a.n_rb, r0 = (pair - h * a.n_rb) * 16;
    const Span sp = span_of(a, b);
    const int sh = a.page_shift + 4;
    int t0 = (sp.start / kPageTile + (x - p0)) * kPageTile;

    // ids of 64 pages, one a lane
    const int32_t* row = a.table + (int64_t)b * a.max_pages;
    int first = t0 >> sh;
    int ids = early;
    const auto list = [&](int t) {
      first = t >> sh;
      ids = first + lane < a.max_pages ? row[first + lane] : -1;
      asm volatile("" : "+v"(ids));    // waited for here: the reads of ids then wait for no tile
    };
    if (!SINGLE || a.window > 0) list(t0);
    else asm volatile("" : "+v"(ids));
    const uint16_t* q = a.q + b * a.q_stride + (int64_t)(h * a.group + r0 + m) * D + 8 * g;
    uint4_t qf[KS];
#pragma unroll
    for (int i = 0; i < KS; ++i) qf[i] = r0 + m < a.group ? *reinterpret_cast<const uint4_t*>(q + 32 * i) : 0;
    // wide heads: the registers are short, so the query waits in the wave's part of LDS, read
    // by offsets from one LDS address (a generic pointer takes two registers for each piece: spills)
    // (what rows past the group read there goes into columns that nobody reads)
    typedef volatile __attribute__((address_space(3))) uint4_t lds_t;
    lds_t* held = (lds_t*)(joined + (wv * a.rows + min(m, a.rows - 1)) * PS) + g;
    if constexpr (D > 192) {
      if (m < a.rows)
#pragma unroll
        for (int i = 0; i < KS; ++i) held[4 * i] = qf[i];
    }

    ref = kNoRef;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < VB; ++i) o[i] = 0.f;

    // where the 16 tokens from t on lie, in elements; -1: nowhere
    const auto place = [&](int t) -> int64_t {
      if (t >= sp.len) return -1;
      const int id = __builtin_amdgcn_readlane(ids, (t >> sh) - first);
      if ((unsigned)id >= (unsigned)a.n_pages) return -1;
      return (((int64_t)id * a.n_kv_heads + h) * (1 << sh) + (t & ((1 << sh) - 1))) * D;
    };
    // Two tiles of registers where they fit (d up to 128): the next tile is on its way
    // while this one is worked on.  Above that, the next keys go where this tile's were
    // once the scores are done, and the next values likewise.
    constexpr int NB = D <= 128 ? 2 : 1;
    uint4_t kf[NB][2][KS], vf[NB][VB];
    int64_t at0, at1;
    const auto find = [&](int t) {
      if (((t + 16) >> sh) - first >= 64) list(t);
      at0 = place(t);
      at1 = place(t + 16);
    };
    const auto fetch = [](const uint16_t* p) { return __builtin_nontemporal_load(reinterpret_cast<const uint4_t*>(p)); };
    const auto load_k = [&](uint4_t (&k)[2][KS]) {
      const uint16_t* k0 = a.k + max(at0, (int64_t)0);
      const uint16_t* k1 = a.k + max(at1, (int64_t)0);
#pragma unroll
      for (int i = 0; i < KS; ++i) k[0][i] = fetch(k0 + (4 * i + g) * 128 + m * 8);
#pragma unroll
      for (int i = 0; i < KS; ++i) k[1][i] = fetch(k1 + (4 * i + g) * 128 + m * 8);
    };
    const auto load_v = [&](uint4_t (&v)[VB]) {
      const uint16_t* v0 = a.v + max(g < 2 ? at0 : at1, (int64_t)0) + (g & 1) * 8 * D + m * 8;
#pragma unroll
      for (int i = 0; i < VB; ++i) v[i] = fetch(v0 + i * 128);
    };

    const auto hide_scores = [&](float (&s)[8], int g, bool here0, bool here1) {
      const int t = t0 + 4 * g;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (!(here0 && t + j >= sp.start && t + j < sp.len)) s[j] = -__builtin_inff();
        if (!(here1 && t + 16 + j >= sp.start && t + 16 + j < sp.len)) s[4 + j] = -__builtin_inff();
      }
    };
    const auto hide_values = [&](auto& v, int g, bool here0, bool here1) {   // nothing of a masked token's counts
      const int t = t0 + 8 * g;
      const bool here = g < 2 ? here0 : here1;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool lo = here && t + 2 * j >= sp.start && t + 2 * j < sp.len;
        const bool hi = here && t + 2 * j + 1 >= sp.start && t + 2 * j + 1 < sp.len;
        const uint32_t keep = (lo ? 0xffffu : 0u) | (hi ? 0xffff0000u : 0u);
#pragma unroll
        for (uint4_t& x : v) x[j] &= keep;
      }
    };
    // the second product's operand: one term of p, which is left with the rest
    const auto operand = [&](float (&p)[8]) {
      uint4_t pf;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t u = take<TY>(p[2 * j], p[2 * j + 1]), w2 = take<TY>(p[4 + 2 * j], p[5 + 2 * j]);
        const auto half = __builtin_amdgcn_permlane32_swap(u, w2, false, false);
        const auto quad = __builtin_amdgcn_permlane16_swap(half[0], half[1], false, false);
        pf[j] = quad[0];
        pf[2 + j] = quad[1];
      }
      return pf;
    };

    const auto step = [&](uint4_t (&k)[2][KS], uint4_t (&v)[VB], uint4_t (&kn)[2][KS], uint4_t (&vn)[VB], bool more) {
      const bool here0 = at0 >= 0, here1 = at1 >= 0;
      const bool whole = here0 && here1 && t0 >= sp.start && t0 + kPageTile <= sp.len;
      if (more) find(t0 + turn * kPageTile);
      if (NB == 2 && more) {
        load_k(kn);
        load_v(vn);
      }
      float4_t s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        uint4_t qi;
        if constexpr (D > 192) qi = held[4 * i];
        else qi = qf[i];
        s0 = product<TY>(k[0][i], qi, s0);
        s1 = product<TY>(k[1][i], qi, s1);
      }
      if (NB == 1 && more) load_k(kn);
      float s[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[j] = s0[j] * a.qscale;
        s[4 + j] = s1[j] * a.qscale;
      }
      if (!whole) hide_scores(s, g, here0, here1);
      float top = s[0];
#pragma unroll
      for (int j = 1; j < 8; ++j) top = fmaxf(top, s[j]);
      if (__ballot(top > ref + kRefMove)) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (top > ref + kRefMove) {
          const float to = top - kRefTop, f = __builtin_amdgcn_exp2f(ref - to);
          ref = to;
          l *= f;
#pragma unroll
          for (int i = 0; i < VB; ++i) o[i] *= f;
        }
      }
      float p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        p[j] = __builtin_amdgcn_exp2f(s[j] - ref);
        l += p[j];
      }
      if (!whole) hide_values(v, g, here0, here1);
#pragma unroll
      for (int term = 0; term < (TY == DWKV_F16 ? 2 : 3); ++term) {
        const uint4_t pf = operand(p);
#pragma unroll
        for (int i = 0; i < VB; ++i) o[i] = product<TY>(v[i], pf, o[i]);
      }
      if (NB == 1 && more) load_v(vn);
      t0 += turn * kPageTile;
    };
    find(t0);
    load_k(kf[0]);
    load_v(vf[0]);
    if constexpr (NB == 2) {
      int i = 0;
      for (; i + 1 < n; i += 2) {
        step(kf[0], vf[0], kf[1], vf[1], true);
        step(kf[1], vf[1], kf[0], vf[0], i + 2 < n);
      }
      if (i < n) step(kf[0], vf[0], kf[1], vf[1], false);
    } else {
      for (int i = 0; i < n; ++i) step(kf[0], vf[0], kf[0], vf[0], i + 1 < n);
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);

    // A weight's later terms may be 0 or below, and the first one 0 where the weight is not: times them an
    // infinite value is NaN.  Sums that are not finite are worked out once more, over the values that
    // are not, with a weight of one for every score above -inf.  Sums of finite values that passed
    // float32's range are kFar meanwhile, and infinite again.  The check costs a wave some 0.1 us:
    // 256 sequences of 64 tokens with 8 KV heads take 30 us, 29.4 without it, longer ones the same.
    float4_t zero = 0.f;
#pragma unroll
    for (int k = 0; k < VB; ++k) zero += o[k] * 0.f;
    const float sign = (zero[0] + zero[1]) + (zero[2] + zero[3]);
    if (__builtin_expect(__ballot(sign != sign && l == l && r0 + m < a.group) != 0, 0)) {
      // a piece at a time, with numbers that are not made before: registers are short, and the loop
      // above needs them
      int id = threadIdx.x;
      float far = kFar;
      asm volatile("" : "+v"(id), "+s"(far));
      const int em = id & 15, eg = (id & 63) >> 4;
#pragma unroll
      for (int k = 0; k < VB; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[k][j] = __builtin_amdgcn_fmed3f(o[k][j], -far, far);
      t0 -= n * turn * kPageTile;
      list(t0);
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        find(t0);
        const bool here0 = at0 >= 0, here1 = at1 >= 0;
        const uint16_t* k0 = a.k + max(at0, (int64_t)0) + eg * 128 + em * 8;
        const uint16_t* k1 = a.k + max(at1, (int64_t)0) + eg * 128 + em * 8;
        const uint16_t* v0 = a.v + max(eg < 2 ? at0 : at1, (int64_t)0) + (eg & 1) * 8 * D + em * 8;
        float4_t s0 = 0.f, s1 = 0.f;
#pragma unroll
        for (int c = 0; c < KS; ++c) {
          uint4_t qi;
          if constexpr (D > 192) qi = held[4 * c];
          else qi = qf[c];
          s0 = product<TY>(fetch(k0 + 512 * c), qi, s0);
          s1 = product<TY>(fetch(k1 + 512 * c), qi, s1);
          asm volatile("" ::: "memory");
        }
        float p[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          p[j] = s0[j] * a.qscale;
          p[4 + j] = s1[j] * a.qscale;
        }
        hide_scores(p, eg, here0, here1);
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = p[j] > -__builtin_inff() ? 1.f : 0.f;
        const uint4_t pf = operand(p);
#pragma unroll
        for (int k = 0; k < VB; ++k) {
          uint4_t v[1] = {fetch(v0 + 128 * k)};
          hide_values(v, eg, here0, here1);
#pragma unroll
          for (int j = 0; j < 4; ++j) v[0][j] = not_finite<TY>(v[0][j]);
          o[k] = product<TY>(v[0], pf, o[k]);
          asm volatile("" ::: "memory");
        }
        t0 += turn * kPageTile;
      }
#pragma unroll
      for (int k = 0; k < VB; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (__builtin_fabsf(o[k][j]) == far) o[k][j] = __builtin_copysignf(__builtin_inff(), o[k][j]);
    }
    if (!join && r0 + m < a.group) {
      if (x == p0 && n == T) {           // a pair of this wave's own
        float* out = a.out + ((int64_t)b * a.n_kv_heads * a.group + h * a.group + r0 + m) * D + 4 * g;
        const bool some = l > 0.f || l != l;
        const float f = some ? 1.f / l : 0.f;
#pragma unroll
        for (int k = 0; k < VB; ++k) *reinterpret_cast<float4_t*>(out + 16 * k) = some ? o[k] * f : float4_t(0.f);
      } else {
        float* part = a.part + ((int64_t)slot_of(w, x, p0) * a.rows + m) * PS;
#pragma unroll
        for (int k = 0; k < VB; ++k) *reinterpret_cast<float4_t*>(part + 16 * k + 4 * g) = o[k];
        if (g == 0) {
          part[D] = ref;
          part[D + 1] = l;
        }
      }
    }
    x += n * turn;
  }
  if (!join) return;

  if (m < a.rows) {
    float* mine = joined + (wv * a.rows + m) * PS;
#pragma unroll
    for (int k = 0; k < VB; ++k) *reinterpret_cast<float4_t*>(mine + 16 * k + 4 * g) = o[k];
    if (g == 0) {
      mine[D] = ref;
      mine[D + 1] = l;
    }
  }
  __syncthreads();
  const int h = wgp / a.n_rb, r0 = (wgp - h * a.n_rb) * 16;
  const bool own = wg0 == wgp0 && wg1 == wgp0 + wgT;
  for (int u = threadIdx.x; u < a.rows * (D / 4); u += kPT) {
    const int r = u / (D / 4), c = (u - r * (D / 4)) * 4;
    if (r0 + r >= a.group) break;
    float top = kNoRef;
    for (int i = 0; i < kPageWaves; ++i) top = fmaxf(top, joined[(i * a.rows + r) * PS + D]);
    float4_t sum = 0.f;
    float all = 0.f;
    for (int i = 0; i < kPageWaves; ++i) {
      const float* from = joined + (i * a.rows + r) * PS;
      const float f = __builtin_amdgcn_exp2f(from[D] - top);
      sum += *reinterpret_cast<const float4_t*>(from + c) * f;
      all += from[D + 1] * f;
    }
    const float4_t zero = sum * 0.f;
    const float sign = (zero[0] + zero[1]) + (zero[2] + zero[3]);
    if (__builtin_expect(sign != sign && all == all, 0)) {
      sum = 0.f;
#pragma unroll 1
      for (int i = 0; i < kPageWaves; ++i) {
        const float* from = joined + (i * a.rows + r) * PS;
        const float f = __builtin_amdgcn_exp2f(from[D] - top);
        for (int j = 0; j < 4; ++j) sum[j] = plus(sum[j], from[c + j], f);
      }
    }
    if (own) {
      const bool some = all > 0.f || all != all;
      *reinterpret_cast<float4_t*>(a.out + ((int64_t)b * a.n_kv_heads * a.group + h * a.group + r0 + r) * D + c) =
          some ? sum * (1.f / all) : float4_t(0.f);
    } else {
      float* part = a.part + ((int64_t)slot_of(blockIdx.x * kPageWaves, wg0, wgp0) * a.rows + r) * PS;
      *reinterpret_cast<float4_t*>(part + c) = sum;
      if (c == 0) {
        part[D] = top;
        part[D + 1] = all;
      }
    }
  }
}

// grid (query heads, B): joins the partials of a pair that several waves shared.  Its
// threads fall into groups of d / 4 that take the partials in turn, each with a
// reference of its own, so that weights and sums are on their way together.
template <int D>
__global__ __launch_bounds__(256) void page_merge_kernel(const PageArgs a) {
  constexpr int PS = D + 4, LN = D / 4, NG = 256 / LN;
  __shared__ float tops[NG], alls[NG];
  __shared__ __align__(16) float sums[NG][D];
  const int b = blockIdx.y, hq = blockIdx.x, h = hq / a.group, r = hq - h * a.group;
  const int pb = a.plan[b], T = a.plan[b + 1] - pb, pairs = a.n_kv_heads * a.n_rb, total = a.plan[a.batch] * pairs;
  float* out = a.out + ((int64_t)b * gridDim.x + hq) * D;
  if (T == 0) {
    if (threadIdx.x < D) out[threadIdx.x] = 0.f;
    return;
  }
  const Share s = share_of(total);
  const int p0 = pb * pairs + (h * a.n_rb + r / 16) * T, p1 = p0 + T;
  const int g0 = p0 / s.wg, g1 = (p1 - 1) / s.wg;
  const int w0 = g0 * kPageWaves + (p0 - g0 * s.wg) / s.per, w1 = g1 * kPageWaves + (p1 - 1 - g1 * s.wg) / s.per;
  if (w0 == w1) return;                                      // written by its wave
  const auto joined = [&](int g) {
    const int x = g * s.wg;
    return x >= p0 && min(total, x + s.wg) <= p1;
  };
  const bool j0 = joined(g0), j1 = joined(g1);
  if (g0 == g1 && j0) return;                                // written by its workgroup
  const int n0 = j0 ? 1 : min(w1, g0 * kPageWaves + (s.wg - 1) / s.per) - w0 + 1, mid = max(0, g1 - g0 - 1);
  const int n = n0 + mid + (g1 == g0 ? 0 : j1 ? 1 : w1 - g1 * kPageWaves + 1);
  const auto partial = [&](int i) -> const float* {
    int slot;
    if (i < n0) slot = j0 ? 2 * g0 * kPageWaves + 1 : 2 * (w0 + i) + (i == 0);
    else if (i < n0 + mid) slot = 2 * (g0 + 1 + i - n0) * kPageWaves;
    else slot = 2 * (g1 * kPageWaves + (i - n0 - mid));
    return a.part + ((int64_t)slot * a.rows + (r & 15)) * PS;
  };
  const int c = threadIdx.x % LN, k = threadIdx.x / LN;
  constexpr int kAt = 4;                                     // partials of a group under way
  float top = kNoRef, all = 0.f;
  float4_t sum = 0.f;
  if (k < NG)
    for (int i0 = k; i0 < n; i0 += kAt * NG) {
      float4_t v[kAt];
      float2 of[kAt];
#pragma unroll
      for (int j = 0; j < kAt; ++j) {
        const float* p = partial(min(i0 + j * NG, n - 1));
        v[j] = *reinterpret_cast<const float4_t*>(p + 4 * c);
        of[j] = *reinterpret_cast<const float2*>(p + D);
      }
      float to = top;
#pragma unroll
      for (int j = 0; j < kAt; ++j)
        if (i0 + j * NG < n) to = fmaxf(to, of[j].x);
      const float f = __builtin_amdgcn_exp2f(top - to);
      sum *= f;
      all *= f;
      top = to;
#pragma unroll
      for (int j = 0; j < kAt; ++j)
        if (i0 + j * NG < n) {
          const float e = __builtin_amdgcn_exp2f(of[j].x - to);
          sum += v[j] * e;
          all += of[j].y * e;
        }
    }
  if (k < NG) {
    *reinterpret_cast<float4_t*>(&sums[k][4 * c]) = sum;
    if (c == 0) {
      tops[k] = top;
      alls[k] = all;
    }
  }
  __syncthreads();
  if (threadIdx.x < D) {
    float to = kNoRef, v = 0.f, l = 0.f;
#pragma unroll
    for (int i = 0; i < NG; ++i) to = fmaxf(to, tops[i]);
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const float e = __builtin_amdgcn_exp2f(tops[i] - to);
      v += sums[i][threadIdx.x] * e;
      l += alls[i] * e;
    }
    if (__builtin_expect(v != v && l == l, 0)) {
      v = 0.f;
#pragma unroll 1
      for (int i = 0; i < n; ++i) v = plus(v, partial(i)[threadIdx.x], __builtin_amdgcn_exp2f(partial(i)[D] - to));
    }
    out[threadIdx.x] = l > 0.f || l != l ? v / l : 0.f;
  }
}

// Whether every pair gets one workgroup: by the longest span that the table or the
// window allows (lengths are the device's: a table with room for more than 4096 tokens takes
// the list whatever the lengths are).  A launch and the merge are saved, about 3 us;
// but one compute unit reads no more than 60 GB/s, so long spans of few pairs are better
// shared out.  With heads of 128, nothing in the caches: 2 pairs of 256, 512 and 1000 tokens
// take 4.7, 7.4 and 11.6 us against 7.2, 7.5 and 7.8; 128 pairs 6.7, 9.7 and 16.6 against
// 10.3, 12.9 and 18.4; 256 of 1000 and 2000 tokens 26 and 49 against 29 and 56.  Then by
// how full the last round of workgroups is: 272 of 512 and 1000 tokens 20 and 34 against
// 22 and 33, 512 of 1000 48 against 53.  From two full rounds on, up to 4096 tokens: 512 pairs 187
// against 194, with lengths spread evenly 102 against 107.  With short spans the list wins
// where pairs are many: of 1, 64, 256 and 512 tokens 512 pairs take 8.6, 9.1, 16.3 and 25.4
// against 9.5, 13.5, 22.3 and 31.9, 1024 pairs 15.4, 16.0, 30.1 and 50.3 against 13.8, 21.7, 36.4
// and 58.5, 2048 pairs 29.1, 29.0, 55.1 and 92.2 against 20.6, 26.0, 56.9 and 96.2; with heads of
// 256 2048 pairs 42, 49, 108 and 182 against 26, 39, 103 and 179.
bool one_workgroup_each(int64_t tiles, int64_t pairs, int d) {
  if (tiles > kSingleTiles) return false;
  const int64_t rounds = (pairs + kPageWG - 1) / kPageWG;
  return pairs >= 2 * kPageWG || tiles * d <= std::max<int64_t>(2048, 8192 * pairs / (kPageWG * rounds));
}

template <int D, int TY>
hipError_t launch_t(PageArgs a, hipStream_t s) {
  const int64_t room = (((int64_t)a.max_pages << (a.page_shift + 4)) + kPageTile - 1) / kPageTile;
  const int64_t most = a.window > 0 ? std::min<int64_t>(room, ((int64_t)a.window + kPageTile - 2) / kPageTile + 1) : room;
  const bool single = one_workgroup_each(most, (int64_t)a.n_kv_heads * a.n_rb * a.batch, D);
  const size_t lds = ((size_t)kPageWaves * a.rows * (D + 4) + (single ? 0 : a.batch + 1)) * sizeof(float);
  if (lds > 64 * 1024) {
    const void* k = single ? (const void*)page_split_kernel<D, TY, true> : (const void*)page_split_kernel<D, TY, false>;
    const hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  if (single) {
    // where not all start at once, and are long enough to matter: 1024 pairs with lengths spread
    // up to 4096 take 196 us, 228 as they come; up to 1000 it would cost 56 against 53
    a.longest_first = a.batch <= kRanked && most * D >= 6144 && (int64_t)a.n_kv_heads * a.n_rb * a.batch > kPageWG;
    hipLaunchKernelGGL((page_split_kernel<D, TY, true>), dim3(a.n_kv_heads * a.n_rb, a.batch), dim3(kPT), lds, s, a);
  } else {
    hipLaunchKernelGGL((page_split_kernel<D, TY, false>), dim3(kPageWG), dim3(kPT), lds, s, a);
    hipLaunchKernelGGL((page_merge_kernel<D>), dim3(a.n_kv_heads * a.group, a.batch), dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(const PageArgs& a, int type, hipStream_t s) {
  return type == DWKV_F16 ? launch_t<D, DWKV_F16>(a, s) : launch_t<D, DWKV_BF16>(a, s);
}

}  // namespace

hipError_t launch_page_decode(const PageArgs& a, int d, int type, hipStream_t s) {
  switch (d) {
    case 32: return launch_d<32>(a, type, s);
    case 64: return launch_d<64>(a, type, s);
    case 96: return launch_d<96>(a, type, s);
    case 128: return launch_d<128>(a, type, s);
    case 160: return launch_d<160>(a, type, s);
    case 192: return launch_d<192>(a, type, s);
    case 224: return launch_d<224>(a, type, s);
    default: return launch_d<256>(a, type, s);
  }
}

}  // namespace dwkv
