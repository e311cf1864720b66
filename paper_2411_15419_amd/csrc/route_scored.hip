// luffy_route_scored and luffy_route_scored_backward: a router with softmax or
// sigmoid scores, a bias for balance, groups of experts and up to eight experts a
// token.
//
// Forward kernels:
//   scored_both    (small calls) scored_gate and scored_choose, 16 tokens a block
//   scored_gate    logits by float32 sums on MFMA, and a bound on their error
//   scored_choose  scores and choices; a token with a deciding gap within the bound is
//                  decided in float64 from exact products; ranks every slot among its
//                  chunk's slots of the same expert and leaves the chunks' counts
//                  (one chunk of tokens: the buckets too)
//   slot_place     bucket offsets and positions; slot_scan, slot_scatter (route.hip) where
//                  the counts do not fit LDS
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ffn.h"
#include "luffy_common.h"
#include "route.h"

namespace luffy {
namespace {

constexpr int kMaxChoices = 8, kMaxGroups = 16;
constexpr int kChooseTok = 32, kChooseWaves = 4;   // of a scored_choose block, at most; a histogram chunk is its tokens
constexpr int kAgainExperts = 4;                   // logits that a wave takes again together
constexpr float kLog2e = 1.44269504088896341f;

struct ScoreArgs {
  const float *bias, *balance;   // [E] or null
  int E, k, score, groups, group_size, top_groups, best, renormalise;
  float scale;
};

template <int DPP>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), DPP, 0xF, 0xF, false));
}
template <int N>
__device__ __forceinline__ float ror16f(float x) {   // by N lanes inside each row of 16
  return __uint_as_float(dpp<0x120 + N>(__float_as_uint(x)));
}
// Every lane of a row of 16 ends with the row's maximum or sum.
__device__ __forceinline__ uint32_t max16(uint32_t x) {
  x = max(x, dpp<0x128>(x));
  x = max(x, dpp<0x124>(x));
  x = max(x, dpp<0x122>(x));
  return max(x, dpp<0x121>(x));
}
__device__ __forceinline__ float sum16(float x) {
  x += ror16f<8>(x);
  x += ror16f<4>(x);
  x += ror16f<2>(x);
  return x + ror16f<1>(x);
}
// The two largest, a >= b, of these lanes' and of those that a DPP control exchanges
// them with.
template <int DPP>
__device__ __forceinline__ void best2_step(uint32_t& a, uint32_t& b) {
  const uint32_t c = dpp<DPP>(a), e = dpp<DPP>(b);
  b = max(min(a, c), max(b, e));
  a = max(a, c);
}

// Order-preserving key of a value (integer maxima fold into their exchanges, float
// ones do not).  Every number's key is above 0; NaN counts as -infinity.
__device__ __forceinline__ uint32_t order_key(float v) {
  if (!(v == v)) v = -INFINITY;
  const uint32_t u = __float_as_uint(v);
  return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t key) {   // (0: -infinity's neighbour, a NaN)
  return __uint_as_float(key ^ (static_cast<uint32_t>(static_cast<int32_t>(~key) >> 31) | 0x80000000u));
}
// The value of a key whose low bits `mask` hold something else: off by less than
// (mask + 1) 2^-23 of itself, infinities as they are.
__device__ __forceinline__ float key_value(uint32_t key, uint32_t mask) {
  return key_value(key & 0x80000000u ? key & ~mask : key | mask);
}
__device__ __forceinline__ float max16f(float x) { return key_value(max16(order_key(x))); }

// Whether a >= b, each known to `rel` of itself and `abs` besides, may be the other way
// round.  A b of -infinity (an expert that is masked out) is below every other a, unless
// abs says that the numbers left float32's range.
__device__ __forceinline__ bool uncertain(float a, float b, float rel, float abs) {
  if (b == -INFINITY) return !(abs < INFINITY);
  return !(a - b > fmaf(rel, fabsf(a) + fabsf(b), 2.0f * abs));
}

// The norm of a row of d values, at most, from their squares' float32 sum: squares
// below float32's normal numbers may be missing from it, 2^-126 each, so that rows of
// about 2^-64 and less have a sum of zero.  (Products of theirs, and sums of those, lose
// as much each: kLost d.  A row of zeros is left with bounds far below any other's.)
constexpr float kLost = 0x1p-124f;
__device__ __forceinline__ float norm_most(float ss, int d) {
  return sqrtf(fmaf(static_cast<float>(d), 0x1p-126f, ss));
}

// Roundings of sums on MFMA, each at most 2^-24 of the products' absolute sum.  A step
// is 16 float32 columns: v_mfma_f32_16x16x4_f32 has the bits of four FMAs in a row, each
// rounded to nearest.  Or 32 bf16 columns: v_mfma_f32_16x16x32_bf16 adds eight products at
// a time and rounds then; bits below 2^-24 of the largest of the eight are cut off before,
// eight times 2^-24 of it at most, so that all steps together lose eight roundings by that.
// (Measured on gfx950 with sums that are led by one product and all kinds of others: 0.97 of
// this at most.)  So that bounds stay small, kChain steps are one chain and the chains'
// sums are added up apart (65536 x 4096 bf16, 64 experts: choices 67 us, 118 with a
// quarter of the columns in one chain; the logits take the same).
constexpr int kChain = 4;
template <bool BF16>
__device__ __forceinline__ float sum_roundings(int steps) {
  return static_cast<float>((BF16 ? 4 * kChain + 8 : 16 * kChain) + (steps + kChain - 1) / kChain);
}

// 1 / (1 + e^-l) times e^-shift, shift <= 0: no overflow for any l.
__device__ __forceinline__ float sigmoid_shifted(float l, float shift) {
  return __builtin_amdgcn_exp2f((fminf(l, 0.f) - shift) * kLog2e) *
         __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-fabsf(l) * kLog2e));
}
__device__ __forceinline__ float sigmoid(float l) {
  const float e = __builtin_amdgcn_exp2f(-fabsf(l) * kLog2e);
  return (l < 0.f ? e : 1.0f) * __builtin_amdgcn_rcpf(1.0f + e);
}

// Choice of one token by the 16 lanes of a row, lane m with the logits l[j] of
// experts 16 j + m (those past E are ignored).  dl bounds the logits' error.  Lane i <
// k ends with the i-th expert and its gate; key[j] is not 0 for the experts of the kept
// groups; `marked` is set for the row where a deciding gap may be of either sign (bit 0:
// between experts, bit 1: between groups):
//   logits         2 dl
//   sigmoid + bias a score moves by at most dl / 4, its evaluation and the sum by
//                  less than 2^-20 (1 + |c|)
//   softmax + bias by at most 2 dl of itself (its own exponential and the sum of
//                  all), evaluation as above
// and 2^-17 (2^-19) of either value for the six (four) low bits of a key that hold the
// expert (group), the lower one being the larger key; the sum of a group's two best
// moves by twice that.
//   A lane sorts its experts once; then the row's largest head is the next choice, and
// its lane goes on to its next: the steps are one chain of exchanges, and its length is
// the time.
template <int NEB, bool SIG, bool GROUPED>
__device__ __forceinline__ void choose16(const float (&l)[NEB], const float (&bal)[NEB], const int (&grp)[NEB],
                                         const ScoreArgs& a, float dl, int& expert, float& gate, uint32_t (&key)[NEB],
                                         uint32_t& marked) {
  const int lane = threadIdx.x & 63, m = lane & 15, row = lane & 48;
  constexpr bool sig = SIG, grouped = GROUPED;
  const bool biased = a.balance != nullptr;
  const bool by_score = grouped && !biased && a.best == 2;   // what groups go by
  float s[NEB], top = 0.f, inv_z = 0.f;
  if constexpr (!sig) {
    uint32_t most = 0;
    float z = 0.f;
#pragma unroll
    for (int j = 0; j < NEB; ++j) most = max(most, 16 * j + m < a.E ? order_key(l[j]) : 0u);
    top = key_value(max16(most));
#pragma unroll
    for (int j = 0; j < NEB; ++j) {
      s[j] = __builtin_amdgcn_exp2f((l[j] - top) * kLog2e);
      z += 16 * j + m < a.E ? s[j] : 0.f;
    }
    inv_z = __builtin_amdgcn_rcpf(sum16(z));
#pragma unroll
    for (int j = 0; j < NEB; ++j) s[j] *= inv_z;
  } else if (biased || by_score) {
#pragma unroll
    for (int j = 0; j < NEB; ++j) s[j] = sigmoid(l[j]);
  }
  const float ds = sig ? fmaf(0.25f, dl, 0x1p-21f) : fmaf(2.0f * inv_z, dl, 0x1p-21f);   // (inv_z: the largest score)
  const float dc = biased ? ds : dl;
#pragma unroll
  for (int j = 0; j < NEB; ++j) key[j] = 16 * j + m < a.E ? order_key(biased ? s[j] + bal[j] : l[j]) : 0u;
  uint32_t bad = 0;
  if constexpr (grouped) {
    // every lane: its experts' groups' values, with the group in the low bits
    const bool two = a.best == 2 && a.group_size > 1;
    const int gs = a.group_size;
    uint32_t gk[NEB], u[NEB];
#pragma unroll
    for (int j = 0; j < NEB; ++j) {
      u[j] = by_score && 16 * j + m < a.E ? order_key(s[j]) : key[j];
      gk[j] = 0;
    }
    auto value_key = [&](uint32_t b1, uint32_t b2, int g) {
      const uint32_t v = two ? order_key(key_value(b1) + key_value(b2)) : b1;
      return (v & ~15u) | static_cast<uint32_t>(15 - g);
    };
    if (gs <= 16 && (gs & (gs - 1)) == 0) {
      // a group is gs neighbouring lanes of one register
#pragma unroll
      for (int j = 0; j < NEB; ++j) {
        uint32_t b1 = u[j], b2 = 0;
        if (gs >= 2) best2_step<0xB1>(b1, b2);     // quad_perm [1, 0, 3, 2]
        if (gs >= 4) best2_step<0x4E>(b1, b2);     // quad_perm [2, 3, 0, 1]
        if (gs >= 8) best2_step<0x141>(b1, b2);    // row_half_mirror
        if (gs >= 16) best2_step<0x140>(b1, b2);   // row_mirror
        if (16 * j + m < a.E) gk[j] = value_key(b1, b2, grp[j]);
      }
    } else {
      for (int g = 0; g < a.groups; ++g) {
        uint32_t b1 = 0, b2 = 0;
#pragma unroll
        for (int j = 0; j < NEB; ++j) {
          const uint32_t v = grp[j] == g ? u[j] : 0u;
          b2 = max(b2, min(b1, v));
          b1 = max(b1, v);
        }
        best2_step<0x128>(b1, b2);
        best2_step<0x124>(b1, b2);
        best2_step<0x122>(b1, b2);
        best2_step<0x121>(b1, b2);
        const uint32_t v = value_key(b1, b2, g);
#pragma unroll
        for (int j = 0; j < NEB; ++j)
          if (grp[j] == g && 16 * j + m < a.E) gk[j] = v;
      }
    }
    uint32_t bound = ~0u, last = ~0u;   // the i-th group's key, and the one before
    for (int i = 0; i <= a.top_groups; ++i) {
      uint32_t best = 0;
      last = bound;
#pragma unroll
      for (int j = 0; j < NEB; ++j) best = max(best, gk[j] < bound ? gk[j] : 0u);
      bound = max16(best);
    }
#pragma unroll
    for (int j = 0; j < NEB; ++j)
      if (gk[j] < last) key[j] = 0;
    const float dg = (a.best == 2 ? 2.0f : 1.0f) * (by_score ? ds : dc);
    bad = uncertain(key_value(last, 15u), key_value(bound, 15u), 0x1p-18f, dg) ? 2u : 0u;
  }
  // the lane's experts, largest key first
  uint32_t head[NEB];
#pragma unroll
  for (int j = 0; j < NEB; ++j) head[j] = key[j] ? (key[j] & ~63u) | static_cast<uint32_t>(63 - 16 * j - m) : 0u;
#pragma unroll
  for (int i = 0; i + 1 < NEB; ++i)
#pragma unroll
    for (int j = 0; j + 1 < NEB - i; ++j) {
      const uint32_t hi = max(head[j], head[j + 1]);
      head[j + 1] = min(head[j], head[j + 1]);
      head[j] = hi;
    }
  uint32_t own = 0;   // lane i: the i-th choice's key; lane k: the first that is left out
  for (int i = 0; i <= a.k; ++i) {
    const uint32_t best = max16(head[0]);
    own = m == i ? best : own;
    const bool taken = head[0] == best;   // (none is left: zeros move up)
#pragma unroll
    for (int j = 0; j + 1 < NEB; ++j) head[j] = taken ? head[j + 1] : head[j];
    head[NEB - 1] = taken ? 0u : head[NEB - 1];
  }
  const uint32_t next = dpp<0x101>(own);   // row_shl: lane i + 1's
  bad |= m < a.k && next && uncertain(key_value(own, 63u), key_value(next, 63u), 0x1p-17f, dc) ? 1u : 0u;
  marked = max16(bad);   // (a group's bit is in every lane)
  expert = 63 - static_cast<int>(own & 63u);
  // gates, from the chosen experts' logits
  float lx = 0.f;
#pragma unroll
  for (int j = 0; j < NEB; ++j) {
    const float v = __shfl(l[j], row | (expert & 15), 64);
    if ((expert >> 4) == j) lx = v;
  }
  if (a.renormalise) {
    const bool mine = m < a.k;
    const float most = key_value(max16(mine ? order_key(lx) : 0u));
    const float p = !mine ? 0.f
                          : sig ? sigmoid_shifted(lx, fminf(most, 0.f)) : __builtin_amdgcn_exp2f((lx - most) * kLog2e);
    gate = a.scale * (p * __builtin_amdgcn_rcpf(sum16(p)));
  } else {
    gate = a.scale * (sig ? sigmoid(lx) : __builtin_amdgcn_exp2f((lx - top) * kLog2e) * inv_z);
  }
}

// Logits of TOK = 16 A tokens a block: four waves, each a quarter of d, on 16-token
// by 16-expert MFMA tiles, two batches of two K steps in flight; the quarters are
// added in LDS.  The rows' and the experts' squared norms come from the same
// fragments (the diagonals of their own Grams): with n roundings in a row (sum_roundings)
// and the joins of the quarters and the bias the error of a logit is at most (n + 5) 2^-24
// |x| |w| (the products' absolute sum is at most |x| |w|), the norms being a little off
// covered by a factor of 1.01 (and norm_most).  The bound goes to bound[t k], a token's
// first gate, for scored_choose.
//   Bounded by the loads' latency where T is small (one token of 1024, 16 experts: 4
// us), by rows from HBM and W from L2 where it is large (65536 x 4096 bf16, 64 experts:
// 176 us, 3.0 TB/s; float32 65536 x 1024, 32: 109 us, 2.5 TB/s, bound by the float32
// products).
template <bool BF16, int A>
__device__ __forceinline__ void gate_block(const void* xv, const void* wv, int T, int d, const ScoreArgs& a,
                                           float* logits, float* bound, float* inv_norm) {
  constexpr int TOK = 16 * A, LD = TOK + 4;
  __shared__ __attribute__((aligned(16))) float part[4][kMaxExperts][LD];
  __shared__ float xsq[4][TOK], wsq[4][kMaxExperts];
  using Elem = std::conditional_t<BF16, uint16_t, float>;
  constexpr int VL = 16 / sizeof(Elem), KS = 4 * VL;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, m = lane & 15, q = lane >> 4;
  const int t0 = blockIdx.x * TOK, E = a.E;
  const Elem* X = static_cast<const Elem*>(xv);
  const Elem* W = static_cast<const Elem*>(wv);
  const int neb = (E + 15) >> 4;
  const int nsteps = d / KS, per = (nsteps + 3) / 4, s_lo = w * per, s_hi = min(nsteps, s_lo + per);
  auto mma = [](const Pack16& p, const Pack16& r, f32x4 c) {
    if constexpr (BF16) {
      return mfma16x16x32(p.v, r.v, c);
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) c = __builtin_amdgcn_mfma_f32_16x16x4f32(p.f[u], r.f[u], c, 0, 0, 0);
      return c;
    }
  };
  {
    f32x4 acc[A][4], tot[A][4], sqx[A], sqw[4];
    const Elem *xrow[A], *wrow[4];
#pragma unroll
    for (int i = 0; i < A; ++i) {
      sqx[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      xrow[i] = X + static_cast<size_t>(min(t0 + 16 * i + m, T - 1)) * d + VL * q;
#pragma unroll
      for (int j = 0; j < 4; ++j) tot[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      sqw[j] = f32x4{0.f, 0.f, 0.f, 0.f};
      wrow[j] = W + static_cast<size_t>(min(16 * j + m, E - 1)) * d + VL * q;
    }
    constexpr int B = 2;
    static_assert(2 * B == kChain, "a turn of the loop is a chain");
    Pack16 xa[2][B][A], wa[2][B][4];
    auto load = [&](int s0, Pack16 (&x)[B][A], Pack16 (&ww)[B][4]) {
#pragma unroll
      for (int u = 0; u < B; ++u) {
        const bool in = s0 + u < s_hi;
#pragma unroll
        for (int i = 0; i < A; ++i)
          x[u][i].u4 = in ? *reinterpret_cast<const uint4*>(xrow[i] + KS * (s0 + u)) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          ww[u][j].u4 = in && j < neb ? *reinterpret_cast<const uint4*>(wrow[j] + KS * (s0 + u))
                                      : make_uint4(0, 0, 0, 0);
      }
    };
    auto compute = [&](const Pack16 (&x)[B][A], const Pack16 (&ww)[B][4], bool first) {
#pragma unroll
      for (int u = 0; u < B; ++u) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (j >= neb) break;
          sqw[j] = mma(ww[u][j], ww[u][j], sqw[j]);
#pragma unroll
          for (int i = 0; i < A; ++i)
            acc[i][j] = mma(x[u][i], ww[u][j], first && u == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[i][j]);
        }
#pragma unroll
        for (int i = 0; i < A; ++i) sqx[i] = mma(x[u][i], x[u][i], sqx[i]);
      }
    };
    if (s_lo < s_hi) load(s_lo, xa[0], wa[0]);
    for (int s0 = s_lo; s0 < s_hi; s0 += 2 * B) {
      if (s0 + B < s_hi) load(s0 + B, xa[1], wa[1]);
      compute(xa[0], wa[0], true);
      if (s0 + B < s_hi) {
        if (s0 + 2 * B < s_hi) load(s0 + 2 * B, xa[0], wa[0]);
        compute(xa[1], wa[1], false);
      }
#pragma unroll
      for (int i = 0; i < A; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < neb) tot[i][j] += acc[i][j];
    }
    // element (m, m) of a 16 x 16 Gram: lane 16 (m / 4) + m, register m % 4
    auto diagonal = [&](const f32x4& g) {
      return (m & 3) == 0 ? g[0] : (m & 3) == 1 ? g[1] : (m & 3) == 2 ? g[2] : g[3];
    };
    if ((m >> 2) == q) {
#pragma unroll
      for (int i = 0; i < A; ++i) xsq[w][16 * i + m] = diagonal(sqx[i]);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < neb) wsq[w][16 * j + m] = diagonal(sqw[j]);
    }
    // the lane holds tokens 16 i + 4 q + r of expert 16 j + m
#pragma unroll
    for (int i = 0; i < A; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < neb) *reinterpret_cast<f32x4*>(&part[w][16 * j + m][16 * i + 4 * q]) = tot[i][j];
  }
  __syncthreads();
  // sixteen lanes a token, lane m experts 16 j + m
  float bias[4], wmost = 0.f, bmost = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int e = 16 * j + m;
    const bool in = e < E;
    bias[j] = in && a.bias ? a.bias[e] : 0.f;
    bmost = fmaxf(bmost, fabsf(bias[j]));
    const float sq = in ? ((wsq[0][e] + wsq[1][e]) + wsq[2][e]) + wsq[3][e] : 0.f;
    wmost = sq > wmost || sq != sq ? sq : wmost;   // NaN stays
  }
  // (a NaN norm marks every token: fmaxf would drop it)
  wmost = __any(wmost != wmost) ? NAN : max16f(wmost);
  bmost = max16f(bmost);
  for (int it = w; it < TOK / 4; it += 4) {
    const int tl = 4 * it + q, t = t0 + tl;
    if (t >= T) continue;
    const float ss = ((xsq[0][tl] + xsq[1][tl]) + xsq[2][tl]) + xsq[3][tl];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int e = 16 * j + m;
      if (e < E)
        logits[static_cast<size_t>(t) * E + e] =
            ((part[0][e][tl] + part[1][e][tl]) + part[2][e][tl]) + part[3][e][tl] + bias[j];
    }
    if (m == 0) {
      bound[static_cast<size_t>(t) * a.k] =
          fmaf(0x1p-23f, bmost, kLost * static_cast<float>(d)) +
          1.01f * (sum_roundings<BF16>(per) + 5.0f) * 0x1p-24f * norm_most(ss, d) * norm_most(wmost, d);
      if (inv_norm) inv_norm[t] = ss > 0.f ? 1.0f / sqrtf(ss) : 0.f;
    }
  }
}

template <bool BF16, int A>
__global__ __launch_bounds__(256) void scored_gate_kernel(const void* __restrict__ xv, const void* __restrict__ wv,
                                                          int T, int d, ScoreArgs a, float* __restrict__ logits,
                                                          float* __restrict__ bound, float* __restrict__ inv_norm) {
  gate_block<BF16, A>(xv, wv, T, d, a, logits, bound, inv_norm);
}

// bf16 logits for W of at most kStreamLds bytes and many tokens: persistent blocks
// hold W in LDS, and every wave takes 16 tokens over the whole of d, 2 NB K steps of
// loads in flight: 8 with 16 waves a block, 16 with up to eight, which have the
// registers for them (about 128 KB a CU either way).
//   Bounded by the rows' stream: 32768 x 2048, 32 experts 41 us (3.3 TB/s; a launch and
// W's staging are 8 of them), 65536 x 1024, 16 experts 32 us (4.1 TB/s).
constexpr int kStreamLds = 128 * 1024, kStreamWaves = 16;

inline bool stream_ok(int dtype, int E, int d) {
  return dtype == LUFFY_BF16 && static_cast<long long>(E) * d * 2 <= kStreamLds;
}

template <int NEB, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void scored_gate_stream_kernel(
    const uint16_t* __restrict__ X, const uint16_t* __restrict__ W, int T, int d, ScoreArgs a,
    float* __restrict__ logits, float* __restrict__ bound, float* __restrict__ inv_norm) {
  // row e's 16-byte chunk c at e * d/8 + (c ^ (e & 7)): the 16 rows that a fragment
  // read touches fall on distinct banks; then the rows' squared norms
  __shared__ __attribute__((aligned(16))) uint8_t lds[kStreamLds + kMaxExperts * 4];
  uint4* wl = reinterpret_cast<uint4*>(lds);
  float* wsq = reinterpret_cast<float*>(lds + kStreamLds);
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, waves = blockDim.x >> 6;
  const int m = lane & 15, q = lane >> 4, E = a.E;
  const int cpr = d >> 3;
  constexpr int NB = WAVES > 8 ? 4 : 8;
  const int nsteps = d >> 5, nchunks = (T + 15) >> 4;
  Pack16 x[2][NB];
  auto load = [&](int ch, int s0, Pack16 (&xx)[NB]) {
    // two steps take 128 bytes of a row: step 2 p has values 64 p + 16 q .. + 7 in
    // lane group q, step 2 p + 1 the eight after them (the sum may take the values
    // in any order), so that both loads of a lane are of one line
    const uint16_t* arow = X + static_cast<size_t>(min(ch * 16 + m, T - 1)) * d + 16 * q;
#pragma unroll
    for (int u = 0; u < NB; ++u)   // (nsteps and s0 are even)
      xx[u].u4 = s0 + u < nsteps ? *reinterpret_cast<const uint4*>(arow + 32 * (s0 + (u & ~1)) + 8 * (u & 1))
                                 : make_uint4(0, 0, 0, 0);
  };
  int ch = blockIdx.x * waves + w;
  load(min(ch, nchunks - 1), 0, x[0]);   // on its way while W is staged
  for (int e = w; e < E; e += waves) {
    float s = 0.f;
    for (int c = lane; c < cpr; c += 64) {
      Pack16 v;
      v.u4 = reinterpret_cast<const uint4*>(W)[static_cast<size_t>(e) * cpr + c];
      wl[e * cpr + (c ^ (e & 7))] = v.u4;
#pragma unroll
      for (int u = 0; u < 8; ++u) s = fmaf(bf16_to_f32(v.h[u]), bf16_to_f32(v.h[u]), s);
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o, 64);
    if (lane == 0) wsq[e] = s;
  }
  int brow[NEB];
  float bias[NEB], bmost = 0.f;
#pragma unroll
  for (int j = 0; j < NEB; ++j) {
    const int e = 16 * j + m, er = min(e, E - 1);
    brow[j] = er * cpr + ((2 * q) ^ (er & 7));   // (the odd step's chunk: its lowest bit flipped)
    bias[j] = e < E && a.bias ? a.bias[e] : 0.f;
    bmost = fmaxf(bmost, fabsf(bias[j]));
  }
  __syncthreads();
  float wmost = 0.f;
#pragma unroll
  for (int j = 0; j < NEB; ++j) {
    const float sq = wsq[min(16 * j + m, E - 1)];
    wmost = sq > wmost || sq != sq ? sq : wmost;
  }
  // (a NaN norm marks every token: fmaxf would drop it)
  wmost = __any(wmost != wmost) ? NAN : max16f(wmost);
  const float rel = 1.01f * (sum_roundings<true>(nsteps) + 2.0f) * 0x1p-24f * norm_most(wmost, d);
  const float add = fmaf(0x1p-23f, max16f(bmost), kLost * static_cast<float>(d));
  for (; ch < nchunks; ch += gridDim.x * waves) {
    const int t0 = ch * 16;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    f32x4 tot[NEB], acc[NEB], sq = zero;
#pragma unroll
    for (int j = 0; j < NEB; ++j) tot[j] = zero;
    auto compute = [&](int s0, const Pack16 (&xx)[NB]) {
#pragma unroll
      for (int u = 0; u < NB; ++u) {
        if (s0 + u >= nsteps) break;
        const int c8 = 4 * (s0 + (u & ~1));
#pragma unroll
        for (int j = 0; j < NEB; ++j) {
          Pack16 b;
          b.u4 = wl[(brow[j] ^ (u & 1)) + c8];
          acc[j] = mfma16x16x32(xx[u].v, b.v, u % kChain == 0 ? zero : acc[j]);
          if (u % kChain == kChain - 1 || (u % 2 == 1 && s0 + u + 1 >= nsteps)) tot[j] += acc[j];
        }
        sq = mfma16x16x32(xx[u].v, xx[u].v, sq);
      }
    };
    for (int s0 = 0; s0 < nsteps; s0 += 2 * NB) {
      if (s0 + NB < nsteps) load(ch, s0 + NB, x[1]);
      compute(s0, x[0]);
      static_assert(NB % kChain == 0, "a batch is whole chains");
      // the next batch, at the end the next chunk's first
      const bool more = s0 + 2 * NB < nsteps;
      load(more ? ch : min(ch + static_cast<int>(gridDim.x) * waves, nchunks - 1), more ? s0 + 2 * NB : 0, x[0]);
      if (s0 + NB < nsteps) compute(s0 + NB, x[1]);
    }
    // register i of tot[j]: token 4 q + i, expert 16 j + m; of the squares, element
    // (4 q + i, 4 q + i) is in lane 4 q + i of row q
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = t0 + 4 * q + i;
      const float ss = __shfl(sq[i], (lane & 48) + 4 * q + i, 64);
      if (t < T) {
#pragma unroll
        for (int j = 0; j < NEB; ++j)
          if (16 * j + m < E) logits[static_cast<size_t>(t) * E + 16 * j + m] = tot[j][i] + bias[j];
        if (m == 0) {
          bound[static_cast<size_t>(t) * a.k] = fmaf(rel, norm_most(ss, d), add);
          if (inv_norm) inv_norm[t] = ss > 0.f ? 1.0f / sqrtf(ss) : 0.f;
        }
      }
    }
  }
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ double wave_max64(double v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = fmax(v, __shfl_xor(v, o, 64));
  return v;
}

// Sums over the wave, and the largest (NaN counts as -infinity), in every lane.
__device__ __forceinline__ float wave_sum(float v) {
  v = sum16(v);
  v += __uint_as_float(static_cast<uint32_t>(
      __builtin_amdgcn_update_dpp(0, static_cast<int>(__float_as_uint(v)), 0x142, 0xA, 0xF, false)));   // row_bcast:15
  v += __uint_as_float(static_cast<uint32_t>(
      __builtin_amdgcn_update_dpp(0, static_cast<int>(__float_as_uint(v)), 0x143, 0xC, 0xF, false)));   // row_bcast:31
  return __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(__float_as_uint(v)), 63)));
}
__device__ __forceinline__ float wave_max(float v) {
  uint32_t u = max16(order_key(v));
  u = max(u, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(u), 0x142, 0xA, 0xF, false)));
  u = max(u, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(u), 0x143, 0xC, 0xF, false)));
  return key_value(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(u), 63)));
}
__device__ __forceinline__ double lane_value(double v, int from) {   // from: the same in every lane
  const uint64_t u = __double_as_longlong(v);
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(u), from);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(u >> 32), from);
  return __longlong_as_double(static_cast<long long>((static_cast<uint64_t>(hi) << 32) | lo));
}

// A lane's share of the float64 products of the row at `row` with the experts ec, over
// columns c_lo .. c_hi - 1.
template <class Elem>
__device__ __forceinline__ void products64(const void* __restrict__ xv, const void* __restrict__ wv, size_t row, int d,
                                           const int (&ec)[kAgainExperts], int c_lo, int c_hi,
                                           double (&s)[kAgainExperts]) {
  constexpr int VL = 16 / sizeof(Elem), NE = kAgainExperts;
  const Elem* x = static_cast<const Elem*>(xv) + row;
#pragma unroll
  for (int j = 0; j < NE; ++j) s[j] = 0.0;
  for (int c = c_lo + (threadIdx.x & 63) * VL; c < c_hi; c += 64 * VL) {
    Pack16 xa, wa[NE];
    xa.u4 = *reinterpret_cast<const uint4*>(x + c);
#pragma unroll
    for (int j = 0; j < NE; ++j)
      wa[j].u4 = *reinterpret_cast<const uint4*>(static_cast<const Elem*>(wv) + static_cast<size_t>(ec[j]) * d + c);
    auto value = [](const Pack16& p, int u) {
      if constexpr (VL == 8) return static_cast<double>(bf16_to_f32(p.h[u]));
      else return static_cast<double>(p.f[u]);
    };
#pragma unroll
    for (int u = 0; u < VL; ++u) {
      const double xd = value(xa, u);
#pragma unroll
      for (int j = 0; j < NE; ++j) s[j] = fma(xd, value(wa[j], u), s[j]);
    }
  }
}

// tok tokens a block: choices by the 16 lanes of a row, four tokens a wave at
// a time; then those whose float32 logits do not tell are decided in float64, and
// waves rank the slots of a choice each.
//   Of an undecided token the logits that another one (or, in a group, another
// group's value) is too close to are taken again from exact products, usually two;
// the others are far enough from every other as they are.  All are where float32 sums
// left their range, and in a second pass where other groups are kept than at first and
// their experts are close too, or where under a softmax with a bias the other logits'
// part in the sum still could turn a choice.  The waves share these products.
//   Bounded by its chains, not by bytes (32768 tokens, 32 experts, k 4: 12 MB): a block
// takes some 4 us for the first choices, and one with an undecided token 2 for which
// logits, 2 for the products and 3 for the decision; 19.8 us in all.  The softmax, the
// sigmoid and the groups are compiled apart (a runtime switch: 2 us more).  One block
// per 64 tokens 23.7 us, eight waves per 32 22.9.
//   T <= tok: the one block has every slot, and lays out the buckets as well.
template <int NEB, bool SIG, bool GROUPED>
__device__ __forceinline__ void choose_block(const void* xv, const void* wv, bool bf16, int T, int d, int tok,
                                             const ScoreArgs& a, int C, int32_t* topk_idx, float* topk_gate,
                                             float* logits, int32_t* slot_pos, int32_t* hist, int* scan_done,
                                             int32_t* perm_token, int32_t* offsets) {
  constexpr int NE = kAgainExperts, ITEMS = 16;
  __shared__ int choice[kMaxChoices][kChooseTok];
  __shared__ int cnt[kMaxChoices][kMaxExperts];
  __shared__ float bounds[kChooseTok];
  __shared__ uint32_t marks[kChooseTok];
  __shared__ uint64_t kepts[kChooseTok];          // experts of a marked token's kept groups
  __shared__ int first[kMaxExperts];              // (one chunk) an expert's first position
  __shared__ uint64_t agains[kChooseTok];         // of the n-th marked token: the logits to take again
  __shared__ double lg[kChooseTok][kMaxExperts];  // a marked token's logits
  __shared__ double vals[kChooseWaves][kMaxExperts], gvals[kChooseWaves][kMaxGroups];
  __shared__ double sums[kChooseWaves][ITEMS][NE];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, m = lane & 15, q = lane >> 4;
  const int ch = blockIdx.x, t0 = ch * tok, E = a.E, k = a.k, nch = gridDim.x, rows = tok / 4 / kChooseWaves;
  constexpr bool sig = SIG, grouped = GROUPED;
  if (ch == 0 && threadIdx.x == 0) *scan_done = 0;   // armed for slot_scan
  {
    float bal[NEB], l[NEB], dl, ahead[NEB], dl_ahead;
    int grp[NEB];
#pragma unroll
    for (int j = 0; j < NEB; ++j) {
      const int e = 16 * j + m;
      bal[j] = e < E && a.balance ? a.balance[e] : 0.f;
      grp[j] = e < E && grouped ? e / a.group_size : 0;
    }
    auto load = [&](int i) {
      const size_t t = min(t0 + 4 * (w + kChooseWaves * i) + q, T - 1);
#pragma unroll
      for (int j = 0; j < NEB; ++j) ahead[j] = logits[t * E + min(16 * j + m, E - 1)];
      dl_ahead = topk_gate[t * k];
    };
    load(0);
    // (not unrolled: the code is fetched once a block, cold)
#pragma unroll 1
    for (int i = 0; i < rows; ++i) {
      const int tl = 4 * (w + kChooseWaves * i) + q, t = t0 + tl;
#pragma unroll
      for (int j = 0; j < NEB; ++j) l[j] = ahead[j];
      dl = dl_ahead;
      if (i + 1 < rows) load(i + 1);
      int expert;
      float gate;
      uint32_t key[NEB], marked;
      choose16<NEB, SIG, GROUPED>(l, bal, grp, a, dl, expert, gate, key, marked);
      if (t >= T) marked = 0;
      if (m < k) {
        choice[m][tl] = expert;
        if (t < T && !marked) {
          topk_idx[static_cast<size_t>(t) * k + m] = expert;
          topk_gate[static_cast<size_t>(t) * k + m] = gate;
        }
      }
      if (m == 0) {
        marks[tl] = marked;
        bounds[tl] = dl;
      }
      if (__any(marked)) {
        uint64_t kept = 0;
#pragma unroll
        for (int j = 0; j < NEB; ++j) {
          kept |= ((__ballot(key[j] != 0) >> (lane & 48)) & 0xFFFFull) << (16 * j);
          lg[tl][16 * j + m] = 16 * j + m < E ? l[j] : -INFINITY;
        }
        if (m == 0) kepts[tl] = kept;
      }
    }
  }
  __syncthreads();
  const uint64_t open = __ballot(lane < tok && marks[lane % kChooseTok] != 0);   // the same in every wave
  const int marked = __popcll(open);
  if (marked) {
    auto nth = [&](int n) {   // the n-th marked token
      uint64_t left = open;
      for (; n > 0; --n) left &= left - 1;
      return __ffsll(static_cast<long long>(left)) - 1;
    };
    const bool in = lane < E;
    const uint64_t full = E == 64 ? ~0ull : (1ull << E) - 1;
    const bool by_score = !a.balance && a.best == 2;   // what groups go by
    const float bal = a.balance && in ? a.balance[lane] : 0.f;
    double* val = vals[w];
    double* gval = gvals[w];
    // values of the groups, in lane g, from those of the experts in the lanes
    auto group_values = [&](double v) {
      __builtin_amdgcn_wave_barrier();
      val[lane] = in && v == v ? v : -INFINITY;
      __builtin_amdgcn_wave_barrier();
      double b1 = -INFINITY, b2 = -INFINITY;
      if (lane < a.groups) {
        for (int u = 0; u < a.group_size; ++u) {
          const double e = val[lane * a.group_size + u];
          b2 = fmax(b2, fmin(b1, e));
          b1 = fmax(b1, e);
        }
        gval[lane] = a.best == 2 && a.group_size > 1 ? b1 + b2 : b1;
      }
      __builtin_amdgcn_wave_barrier();
      return a.best == 2 && a.group_size > 1 ? b1 + b2 : b1;
    };
    // which logits to take again
    for (int n = w; n < marked; n += kChooseWaves) {
      const int tl = nth(n);
      const float lf = in ? static_cast<float>(lg[tl][lane % (16 * NEB)]) : -INFINITY, dl = bounds[tl];
      uint64_t again = full;
      if (dl < 0x1p-6f && !__any(in && !(fabsf(lf) < INFINITY))) {
        float top = 0.f, z = 1.f, s = 0.f, ds = 0.f;
        if constexpr (!sig) {
          top = wave_max(lf);
          z = wave_sum(in ? __builtin_amdgcn_exp2f((lf - top) * kLog2e) : 0.f);
          s = __builtin_amdgcn_exp2f((lf - top) * kLog2e) / z;
          ds = fmaf(2.0f / z, dl, 0x1p-20f);
        } else {
          s = sigmoid(lf);
          ds = fmaf(0.25f, dl, 0x1p-20f);
        }
        const float c = a.balance ? s + bal : lf, dc = a.balance ? ds : dl;
        // experts too close to one of the first choice's (an expert that is close to
        // none of those is not among the k best, or surely so and in its place)
        const float close = fmaf(0x1p-15f, wave_max(in && c > -INFINITY ? fabsf(c) : 0.f), 2.0f * dc);
        again = 0;
        for (int j = 0; j < k; ++j) {
          const int e = __builtin_amdgcn_readfirstlane(choice[j][tl]);
          const float v = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(c), e));
          const uint64_t near = __ballot(in && lane != e && fabsf(c - v) <= close);
          if (near) again |= near | (1ull << e);
        }
        if (grouped && (marks[tl] & 2u)) {
          const double g = group_values(by_score ? s : c);
          const double dg = 2.0 * (a.best == 2 ? 2.0 : 1.0) * (by_score ? ds : dc);
          bool hard = false;
          for (int h = 0; h < a.groups; ++h)
            hard = hard || (lane < a.groups && h != lane &&
                            !(fabs(g - gval[h]) > dg + 0x1p-17 * (fabs(g) + fabs(gval[h]))) &&
                            !(g == -INFINITY && gval[h] == -INFINITY));
          const uint64_t groups = __ballot(hard);
          again |= __ballot(in && ((groups >> (in ? lane / a.group_size : 0)) & 1ull));
        }
      }
      if (lane == 0) agains[n] = again;
    }
    __syncthreads();
    for (int pass = 0; pass < 2; ++pass) {
      // their products, NE experts of a token at a time, ITEMS such sums between two
      // barriers; where there are few, the waves take a quarter of d each
      int items = 0;
      for (int n = 0; n < marked; ++n) items += (__popcll(agains[n]) + NE - 1) / NE;
      if (!items) break;   // (the second pass: none was left)
      const bool split = items < 2 * kChooseWaves;
      const int quarter = (d / 8 + kChooseWaves - 1) / kChooseWaves * 8;
      const int c_lo = split ? w * quarter : 0, c_hi = split ? min(d, c_lo + quarter) : d;
      for (int base = 0; base < items; base += ITEMS) {
        int item = 0;
        for (int n = 0; n < marked; ++n) {
          for (uint64_t todo = agains[n]; todo; ++item) {
            int ec[NE];
#pragma unroll
            for (int j = 0; j < NE; ++j) {
              ec[j] = todo ? __ffsll(static_cast<long long>(todo)) - 1 : ec[0];
              todo &= todo - 1;
            }
            if (item < base || item >= base + ITEMS || (!split && item % kChooseWaves != w)) continue;
            double s[NE];
            const size_t row = static_cast<size_t>(t0 + nth(n)) * d;
            if (bf16) products64<uint16_t>(xv, wv, row, d, ec, c_lo, c_hi, s);
            else products64<float>(xv, wv, row, d, ec, c_lo, c_hi, s);
            // four sums over the wave: halves keep two each, quarters one
            static_assert(NE == 4, "four sums a wave");
            const bool h5 = lane & 32, h4 = lane & 16;
            const double p0 = (h5 ? s[2] : s[0]) + __shfl_xor(h5 ? s[0] : s[2], 32, 64);
            const double p1 = (h5 ? s[3] : s[1]) + __shfl_xor(h5 ? s[1] : s[3], 32, 64);
            double sum = (h4 ? p1 : p0) + __shfl_xor(h4 ? p0 : p1, 16, 64);
#pragma unroll
            for (int o = 8; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
            if ((lane & 15) == 0) sums[split ? w : 0][item - base][lane >> 4] = sum;
          }
        }
        __syncthreads();
        // a sum's four quarters, a thread each: the expert and the token again by the
        // same walk
        int at = 0;
        for (int n = 0; n < marked; ++n) {
          const uint64_t mask = agains[n];
          const int below = __popcll(mask & lanemask_lt());   // of this lane's expert
          const int mine = at + below / NE;
          if (w == 0 && ((mask >> lane) & 1ull) && mine >= base && mine < base + ITEMS) {
            double s = sums[0][mine - base][below % NE];
            for (int v = 1; split && v < kChooseWaves; ++v) s += sums[v][mine - base][below % NE];
            lg[nth(n)][lane] = s + (a.bias ? static_cast<double>(a.bias[lane]) : 0.0);
          }
          at += (__popcll(mask) + NE - 1) / NE;
        }
        __syncthreads();
      }
      // the decisions
      for (int n = w; n < marked; n += kChooseWaves) {
        if (pass == 1 && !agains[n]) continue;
        const int tl = nth(n);
        const size_t t = t0 + tl;
        const double l = in ? lg[tl][lane] : -INFINITY;
        double s = 0.0;
        if (a.balance || (grouped && by_score)) {
          if (sig) {
            s = 1.0 / (1.0 + exp(-l));
          } else {
            const double top = wave_max64(l), p = in ? exp(l - top) : 0.0;
            s = p / wave_sum64(p);
          }
        }
        double c = a.balance ? s + static_cast<double>(bal) : l;
        if (!(c == c) || !in) c = -INFINITY;
        // under a softmax with a bias the other logits still move the scores by their
        // sum: by as much of themselves
        const bool moves = pass == 0 && !sig && a.balance && agains[n] != full;
        const double part = moves ? 1.01 * bounds[tl] + 1e-12 : 0.0, s_most = moves ? wave_max64(s) : 0.0;
        bool loose = false;
        uint64_t allowed = kepts[tl];
        if (grouped && ((marks[tl] & 2u) || agains[n] == full)) {
          const double g = group_values(by_score ? s : c);
          int rank = kMaxGroups;
          if (lane < a.groups) {
            rank = 0;
            for (int h = 0; h < a.groups; ++h) {
              rank += gval[h] > g || (gval[h] == g && h < lane);
              loose = loose || (moves && h != lane && fabs(gval[h] - g) <= 2.0 * s_most * part);
            }
          }
          const uint64_t kept = __ballot(rank < a.top_groups);
          allowed = __ballot(in && ((kept >> (in ? lane / a.group_size : 0)) & 1ull));
        }
        // the k best are among the first choice and what was taken again; where other
        // groups are kept than at first, anywhere in them
        const bool turned = allowed != kepts[tl] && agains[n] != full;
        uint64_t may = allowed;
        if (!turned) {
          uint64_t first_choice = 0;
          for (int j = 0; j < k; ++j) first_choice |= 1ull << __builtin_amdgcn_readfirstlane(choice[j][tl]);
          may &= first_choice | agains[n];
        }
        int rank = 0;
        for (uint64_t left = may; left; left &= left - 1) {
          const int e = __builtin_amdgcn_readfirstlane(__ffsll(static_cast<long long>(left)) - 1);
          const double v = lane_value(c, e);
          rank += v > c || (v == c && e < lane);
          if (moves)
            loose = loose || (((may >> lane) & 1ull) && e != lane &&
                              fabs(v - c) <= fabs(lane_value(s, e) - s) * part + 1e-14);
        }
        const bool chosen = ((may >> lane) & 1ull) && rank < k;
        if (turned) {   // gaps to float32 logits: are they wide enough?
          const double dl = bounds[tl], gap = 2.0 * (!a.balance ? dl : sig ? 0.25 * dl : 2.0 * dl) + 1e-12;
          for (uint64_t left = may; left; left &= left - 1) {
            const int e = __builtin_amdgcn_readfirstlane(__ffsll(static_cast<long long>(left)) - 1);
            const bool exact = (agains[n] >> e) & (agains[n] >> lane) & 1ull;
            loose = loose || (chosen && e != lane && !exact && fabs(lane_value(c, e) - c) <= gap);
          }
        }
        const bool all = __any(loose);
        if (lane == 0) agains[n] = all ? full : 0ull;   // none: done
        if (all) continue;
        // gates by choose16's formulas, in float32
        const float lx = static_cast<float>(l);
        const bool of = a.renormalise ? chosen : in;   // what the sum goes over
        float p = 0.f;
        if constexpr (sig) {
          const float shift = a.renormalise ? fminf(wave_max(of ? lx : -INFINITY), 0.f) : 0.f;
          p = in ? sigmoid_shifted(lx, shift) : 0.f;
          if (a.renormalise) p /= wave_sum(of ? p : 0.f);
        } else {
          const float top = wave_max(of ? lx : -INFINITY);
          p = of ? __builtin_amdgcn_exp2f((lx - top) * kLog2e) : 0.f;
          p /= wave_sum(p);
        }
        if (chosen) {
          choice[rank][tl] = lane;
          topk_idx[t * k + rank] = lane;
          topk_gate[t * k + rank] = a.scale * p;
        }
        if (in) logits[t * E + lane] = lx;
      }
      __syncthreads();
    }
  }
  // stable ranks among the chunk's slots of the same expert: the lanes that hold
  // it, by ballots on its bits
  const bool valid = lane < tok && t0 + lane < T;
  constexpr int PER = kMaxChoices / kChooseWaves;
  int ranks[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = w + i * kChooseWaves;
    if (j >= k) break;
    const int e = choice[j][lane % kChooseTok];
    const int key = valid ? e : 127;
    uint64_t same = ~0ull;
#pragma unroll
    for (int b = 0; b < 7; ++b) {
      const bool bit = (key >> b) & 1;
      const uint64_t bb = __ballot(bit);
      same &= bit ? bb : ~bb;
    }
    ranks[i] = __popcll(same & lanemask_lt());
    cnt[j][lane] = 0;
    __builtin_amdgcn_wave_barrier();
    if (valid && ranks[i] == 0) cnt[j][e] = __popcll(same);
    __builtin_amdgcn_wave_barrier();
    if (nch > 1) {
      if (lane < E) hist[static_cast<size_t>(lane) * k * nch + static_cast<size_t>(j) * nch + ch] = cnt[j][lane];
      if (valid) slot_pos[static_cast<size_t>(t0 + lane) * k + j] = ranks[i];
    }
  }
  if (nch > 1) return;
  __syncthreads();
  // the only chunk: an expert a lane, its slots before choice j in cnt[j]
  int total = 0;
  if (w == 0) {
    for (int j = 0; j < k; ++j) {
      const int n = cnt[j][lane];
      cnt[j][lane] = total;
      total += n;
    }
    if (C > 0 && total > C) total = C;
    if (lane >= E) total = 0;
    int incl = total;
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) {
      const int u = __shfl_up(incl, sh, 64);
      if (lane >= sh) incl += u;
    }
    if (lane < E) offsets[lane] = incl - total;
    if (lane == E - 1) offsets[E] = incl;
    first[lane] = incl - total;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = w + i * kChooseWaves;
    if (j >= k) break;
    if (!valid) continue;
    const int e = choice[j][lane % kChooseTok], at = cnt[j][e] + ranks[i];
    const bool kept = C <= 0 || at < C;
    slot_pos[static_cast<size_t>(lane) * k + j] = kept ? first[e] + at : -1;
    if (kept) perm_token[first[e] + at] = lane;
  }
}

template <int NEB, bool SIG, bool GROUPED>
__global__ __launch_bounds__(kChooseWaves * 64) void scored_choose_kernel(
    const void* __restrict__ xv, const void* __restrict__ wv, bool bf16, int T, int d, int tok, ScoreArgs a, int C,
    int32_t* __restrict__ topk_idx, float* __restrict__ topk_gate, float* __restrict__ logits,
    int32_t* __restrict__ slot_pos, int32_t* __restrict__ hist, int* __restrict__ scan_done,
    int32_t* __restrict__ perm_token, int32_t* __restrict__ offsets) {
  choose_block<NEB, SIG, GROUPED>(xv, wv, bf16, T, d, tok, a, C, topk_idx, topk_gate, logits, slot_pos, hist, scan_done,
                                  perm_token, offsets);
}

// Both in one launch, 16 tokens a block (up to 16: the buckets as well).  No pointer is
// __restrict__: the logits and bounds are read back.  Bounded by a launch and its chains:
// one token of 1024 on 16 experts 11.4 us a call, 14.4 in two launches.
template <bool BF16, int NEB, bool SIG, bool GROUPED>
__global__ __launch_bounds__(256) void scored_both_kernel(const void* xv, const void* wv, int T, int d, ScoreArgs a,
                                                           int C, int32_t* topk_idx, float* topk_gate, float* logits,
                                                           float* inv_norm, int32_t* slot_pos, int32_t* hist,
                                                           int* scan_done, int32_t* perm_token, int32_t* offsets) {
  static_assert(kChooseWaves == 4, "the logits' block and the choices' are one");
  gate_block<BF16, 1>(xv, wv, T, d, a, logits, topk_gate, inv_norm);
  __threadfence_block();
  __syncthreads();
  choose_block<NEB, SIG, GROUPED>(xv, wv, BF16, T, d, 16, a, C, topk_idx, topk_gate, logits, slot_pos, hist, scan_done,
                                  perm_token, offsets);
}

// Bucket offsets, positions and tokens in one launch where the chunks' counts (layout:
// RouteWs) fit LDS: every block scans them all by itself, a wave an expert, and takes
// 1024 slots.  Bounded by the chain of trips to memory and the scan (us of a whole call in
// a graph, against slot_scan and slot_scatter: 40 x 1024, 16 experts 10.4 | 14.1, 300 x
// 1024, 64 experts 22.2 | 23.6, 3001 x 512 float32, 8 experts 18.4 | 20.5, 4090 x 1024, 16
// experts, at the limit, 20.5 | 20.4); from the host a launch less is 2.5 more.
constexpr int kPlaceCounts = 16384;

__global__ __launch_bounds__(1024) void slot_place_kernel(const int32_t* __restrict__ topk_idx,
                                                          const int32_t* __restrict__ hist, int T, int k, int E, int C,
                                                          int tok, int32_t* __restrict__ slot_pos,
                                                          int32_t* __restrict__ perm_token,
                                                          int32_t* __restrict__ offsets) {
  __shared__ int cnt[kPlaceCounts];
  __shared__ int totals[kMaxExperts], first[kMaxExperts];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int nblk = (T + tok - 1) / tok, nch = k * nblk, n = E * nch;
  const int s = blockIdx.x * 1024 + tid;   // (E k T / tok counts: a grid of few blocks)
  const bool valid = s < T * k;
  const int j = valid ? s / T : 0, t = valid ? s - j * T : 0;
  const size_t o = static_cast<size_t>(t) * k + j;
  const int e = topk_idx[o], rank = slot_pos[o];
#pragma unroll 4
  for (int i = tid; i < n; i += 1024) cnt[i] = hist[i];
  __syncthreads();
  for (int x = w; x < E; x += 16) {
    int* c = cnt + x * nch;
    int carry = 0;
    for (int c0 = 4 * lane; c0 - 4 * lane < nch; c0 += 256) {
      int v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = c0 + u < nch ? c[c0 + u] : 0;
      const int own = (v[0] + v[1]) + (v[2] + v[3]);
      int incl = own;
#pragma unroll
      for (int sh = 1; sh < 64; sh <<= 1) {
        const int u = __shfl_up(incl, sh, 64);
        if (lane >= sh) incl += u;
      }
      int run = carry + incl - own;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (c0 + u < nch) c[c0 + u] = run;
        run += v[u];
      }
      carry += __builtin_amdgcn_readlane(incl, 63);
    }
    if (lane == 0) totals[x] = carry;
  }
  __syncthreads();
  if (w == 0) {
    int own = lane < E ? totals[lane] : 0;
    if (C > 0 && own > C) own = C;
    int incl = own;
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) {
      const int u = __shfl_up(incl, sh, 64);
      if (lane >= sh) incl += u;
    }
    first[lane] = incl - own;
    if (blockIdx.x == 0) {
      if (lane < E) offsets[lane] = incl - own;
      if (lane == E - 1) offsets[E] = incl;
    }
  }
  __syncthreads();
  if (!valid) return;
  const int pos = cnt[e * nch + j * nblk + t / tok] + rank;
  if (C > 0 && pos >= C) {
    slot_pos[o] = -1;
  } else {
    slot_pos[o] = first[e] + pos;
    perm_token[first[e] + pos] = t;
  }
}

// ---------------------------------------------------------------- backward
// dl, the logits' gradient: with r_j = s_j / sum of the chosen (shifted as in the
// forward, so that nothing under- or overflows)
//   renormalised       dl_j = scale r_j (dg_j - sum_i dg_i r_i), times 1 - s_j for
//                      sigmoid scores; 0 for experts not chosen
//   sigmoid            dl_j = scale dg_j s_j (1 - s_j)
//   softmax            dl_e = s_e (ds_e - sum_i ds_i s_i), ds_j = scale dg_j
// plus what the caller adds.  Sixteen lanes a token, four experts a lane (4 m ..).
//   dl leaves as three bf16 parts (their sum has dl's 24 bits): part p of expert e in
// column p E + e of the rows that scored_dw's product takes.
// db: a lane's sums over its tokens, added up over the block, in a fixed order.
//   Bounded by latency (a token is a chain of loads and row sums): 65536 tokens, 64
// experts, k 8: 17 us for 46 MB.
constexpr int kDlThreads = 256;

template <bool EVEN>   // E is a multiple of 4
__global__ __launch_bounds__(kDlThreads) void scored_dlogits_kernel(
    const float* __restrict__ logits, const int32_t* __restrict__ topk_idx, const float* __restrict__ dgate,
    const float* __restrict__ extra, int T, ScoreArgs a, int ld, uint16_t* __restrict__ dl, int parts, int per,
    int32_t* __restrict__ part_rows, float* __restrict__ part_b) {
  __shared__ float sums[kDlThreads / 16][kMaxExperts];
  const int m = threadIdx.x & 15, E = a.E, k = a.k;
  const bool sig = a.score == LUFFY_SCORE_SIGMOID;
  if (blockIdx.x == 0 && threadIdx.x <= parts) part_rows[threadIdx.x] = min(T, static_cast<int>(threadIdx.x) * per);
  float db[4] = {0.f, 0.f, 0.f, 0.f};
  for (long long t0 = static_cast<long long>(blockIdx.x) * (kDlThreads / 16); t0 < T;
       t0 += static_cast<long long>(gridDim.x) * (kDlThreads / 16)) {
    const long long tt = t0 + threadIdx.x / 16;
    const bool valid = tt < T;
    const size_t t = valid ? tt : T - 1;
    float l[4], ex[4] = {0.f, 0.f, 0.f, 0.f};
    if constexpr (EVEN) {
      const float4 v = 4 * m < E ? *reinterpret_cast<const float4*>(logits + t * E + 4 * m)
                                 : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      l[0] = v.x; l[1] = v.y; l[2] = v.z; l[3] = v.w;
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) l[u] = 4 * m + u < E ? logits[t * E + 4 * m + u] : -INFINITY;
    }
    if (extra)
#pragma unroll
      for (int u = 0; u < 4; ++u) ex[u] = 4 * m + u < E ? extra[t * E + 4 * m + u] : 0.f;
    // lane j < k: the token's j-th choice
    const int idx = m < k ? topk_idx[t * k + m] : -1;
    const float dgj = m < k ? dgate[t * k + m] : 0.f;
    float dg[4] = {0.f, 0.f, 0.f, 0.f};   // of this lane's experts, 0 if not chosen
    bool chosen[4] = {false, false, false, false};
    auto take = [&](uint32_t e, uint32_t g) {
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (static_cast<int>(e) == 4 * m + u) {
          dg[u] += __uint_as_float(g);
          chosen[u] = true;
        }
    };
    const uint32_t iu = static_cast<uint32_t>(idx), gu = __float_as_uint(dgj);
    // (row_newbcast: lane j of each row; lanes from k on hold no expert)
    take(dpp<0x150>(iu), dpp<0x150>(gu));
    take(dpp<0x151>(iu), dpp<0x151>(gu));
    if (k > 2) {
      take(dpp<0x152>(iu), dpp<0x152>(gu));
      take(dpp<0x153>(iu), dpp<0x153>(gu));
    }
    if (k > 4) {
      take(dpp<0x154>(iu), dpp<0x154>(gu));
      take(dpp<0x155>(iu), dpp<0x155>(gu));
      take(dpp<0x156>(iu), dpp<0x156>(gu));
      take(dpp<0x157>(iu), dpp<0x157>(gu));
    }
    float g[4];
    if (a.renormalise) {
      float top = -INFINITY;
#pragma unroll
      for (int u = 0; u < 4; ++u) top = fmaxf(top, chosen[u] ? l[u] : -INFINITY);
      top = max16f(top);
      const float shift = sig ? fminf(top, 0.f) : top;
      float p[4], sum = 0.f, dot = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        p[u] = !chosen[u] ? 0.f : sig ? sigmoid_shifted(l[u], shift) : __builtin_amdgcn_exp2f((l[u] - shift) * kLog2e);
        sum += p[u];
        dot = fmaf(p[u], dg[u], dot);
      }
      const float inv = 1.0f / sum16(sum), mean = sum16(dot) * inv;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        g[u] = chosen[u] ? a.scale * (p[u] * inv) * (dg[u] - mean) : 0.f;
        if (sig && chosen[u]) g[u] *= sigmoid(-l[u]);
      }
    } else if (sig) {
#pragma unroll
      for (int u = 0; u < 4; ++u) g[u] = chosen[u] ? a.scale * dg[u] * (sigmoid(l[u]) * sigmoid(-l[u])) : 0.f;
    } else {
      float top = fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3]));
      top = max16f(top);
      float p[4], sum = 0.f, dot = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        p[u] = __builtin_amdgcn_exp2f((l[u] - top) * kLog2e);
        sum += p[u];
        dot = fmaf(p[u], dg[u], dot);
      }
      const float inv = 1.0f / sum16(sum), mean = sum16(dot) * inv;
#pragma unroll
      for (int u = 0; u < 4; ++u) g[u] = a.scale * (p[u] * inv) * (dg[u] - mean);
    }
    if (!valid) continue;
    uint16_t part[3][4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      float v = 4 * m + u < E ? g[u] + ex[u] : 0.f;
      db[u] += v;
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        const uint32_t b = pack_bf16x2(v, 0.f) & 0xFFFFu;
        part[q][u] = static_cast<uint16_t>(b);
        v -= __uint_as_float(b << 16);
      }
    }
    uint16_t* out = dl + t * ld + 4 * m;
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      if constexpr (EVEN) {
        if (4 * m < E)
          *reinterpret_cast<uint2*>(out + q * E) =
              make_uint2(part[q][0] | static_cast<uint32_t>(part[q][1]) << 16,
                         part[q][2] | static_cast<uint32_t>(part[q][3]) << 16);
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (4 * m + u < E) out[q * E + u] = part[q][u];
      }
    }
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) sums[threadIdx.x / 16][4 * m + u] = db[u];
  __syncthreads();
  if (threadIdx.x < E) {
    float s = 0.f;
    for (int i = 0; i < kDlThreads / 16; ++i) s += sums[i][threadIdx.x];
    part_b[static_cast<size_t>(blockIdx.x) * E + threadIdx.x] = s;
  }
}

// dl from its three parts.
__device__ __forceinline__ float dl_value(const uint16_t* p, int E) {
  return (bf16_to_f32(p[0]) + bf16_to_f32(p[E])) + bf16_to_f32(p[2 * E]);
}

// dx of a token (or of some of its columns) a wave: its experts' rows of W by dl (from
// L2), and the representatives' rows of dx_rep that are this token's, added in float32
// and rounded once.  Bounded by the gathered rows: 65536 x 1024 bf16, k 8, 196 us for 765
// MB, 3.9 TB/s (a large copy 4.9).  Sixteen loads in flight, held in arrays, took 151
// registers and 369 us.
template <bool BF16>
__global__ __launch_bounds__(256) void scored_dx_kernel(const void* __restrict__ wv, const uint16_t* __restrict__ dl,
                                                        int ld, int T, int d, int E, int k, int slices,
                                                        const void* __restrict__ dx_rep,
                                                        const int32_t* __restrict__ slot_pos,
                                                        const int32_t* __restrict__ rep_of_pos,
                                                        const int32_t* __restrict__ rep_row, void* __restrict__ dx) {
  using Elem = std::conditional_t<BF16, uint16_t, float>;
  constexpr int VL = 16 / sizeof(Elem);
  const int lane = threadIdx.x & 63;
  auto unpack = [](const Elem* p, float (&f)[VL]) {
    Pack16 v;
    v.u4 = *reinterpret_cast<const uint4*>(p);
#pragma unroll
    for (int u = 0; u < VL; ++u) {
      if constexpr (BF16) f[u] = bf16_to_f32(v.h[u]);
      else f[u] = v.f[u];
    }
  };
  for (long long i = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 6);
       i < static_cast<long long>(T) * slices; i += static_cast<long long>(gridDim.x) * 4) {
    const long long t = slices == 1 ? i : i / slices;
    const int slice = static_cast<int>(i - t * slices);
    const float g = lane < E ? dl_value(dl + t * ld + lane, E) : 0.f;
    const uint64_t used = __ballot(g != 0.f);
    int row = -1;
    if (dx_rep && lane < k) {
      const int p = slot_pos[t * k + lane];
      if (p >= 0 && rep_of_pos[p] == p) row = rep_row[p];
    }
    // (the lanes past d go along with the last columns)
    for (int c = (64 * slice + lane) * VL; c < (d + 64 * VL - 1) / (64 * VL) * (64 * VL); c += 64 * VL * slices) {
      const int cc = min(c, d - VL);
      float acc[VL], f[VL];
#pragma unroll
      for (int u = 0; u < VL; ++u) acc[u] = 0.f;
      for (uint64_t left = used; left; left &= left - 1) {
        const int e = __ffsll(static_cast<long long>(left)) - 1;
        const float ge = __shfl(g, e, 64);
        unpack(static_cast<const Elem*>(wv) + static_cast<size_t>(e) * d + cc, f);
#pragma unroll
        for (int u = 0; u < VL; ++u) acc[u] = fmaf(ge, f[u], acc[u]);
      }
      for (int j = 0; dx_rep && j < k; ++j) {
        const int r = __shfl(row, j, 64);
        if (r < 0) continue;
        unpack(static_cast<const Elem*>(dx_rep) + static_cast<size_t>(r) * d + cc, f);
#pragma unroll
        for (int u = 0; u < VL; ++u) acc[u] += f[u];
      }
      if (c >= d) continue;
      if constexpr (BF16) {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(dx) + t * d + c) =
            make_uint4(pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3]), pack_bf16x2(acc[4], acc[5]),
                       pack_bf16x2(acc[6], acc[7]));
      } else {
        *reinterpret_cast<float4*>(static_cast<float*>(dx) + t * d + c) = make_float4(acc[0], acc[1], acc[2], acc[3]);
      }
    }
  }
}

constexpr int kDwTok = 64, kDwCols = 64;
constexpr int kMaxDwParts = 64;   // (the product's groups)

// float32 rows: part of dW = dl^T x, 64 columns by the tokens of part blockIdx.y,
// every expert; 64 tokens at a time in LDS, 16 experts a wave, a column a lane.
// (bf16 rows go through the FFN's weight-gradient product, ffn.h: dl's three bf16 parts
// are 3 E of its columns, so the sums are float32's at the matrix cores' rate.  65536 x
// 1024, 64 experts: 44 us, where these products took 260.)
__global__ __launch_bounds__(256) void scored_dw_kernel(const float* __restrict__ xv, const uint16_t* __restrict__ dl,
                                                        int ld, int T, int d, int E, int per,
                                                        float* __restrict__ part_w) {
  __shared__ __attribute__((aligned(16))) float xs[kDwTok][kDwCols], gs[kDwTok][kMaxExperts];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c0 = blockIdx.x * kDwCols;
  const int t_lo = blockIdx.y * per, t_hi = min(T, t_lo + per);
  float acc[16];
#pragma unroll
  for (int u = 0; u < 16; ++u) acc[u] = 0.f;
  for (int t0 = t_lo; t0 < t_hi; t0 += kDwTok) {
    __syncthreads();
    for (int i = threadIdx.x; i < kDwTok * kDwCols / 4; i += 256) {
      const int tl = i / (kDwCols / 4), c = i % (kDwCols / 4) * 4;
      *reinterpret_cast<float4*>(&xs[tl][c]) =
          t0 + tl < t_hi ? *reinterpret_cast<const float4*>(xv + static_cast<size_t>(t0 + tl) * d + c0 + c)
                         : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    for (int i = threadIdx.x; i < kDwTok * kMaxExperts; i += 256) {
      const int tl = i / kMaxExperts, e = i % kMaxExperts;
      gs[tl][e] = t0 + tl < t_hi && e < E ? dl_value(dl + static_cast<size_t>(t0 + tl) * ld + e, E) : 0.f;
    }
    __syncthreads();
    for (int tl = 0; tl < kDwTok; ++tl) {
      const float x = xs[tl][lane];
      const float4* g4 = reinterpret_cast<const float4*>(&gs[tl][16 * w]);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float4 g = g4[u];
        acc[4 * u] = fmaf(g.x, x, acc[4 * u]);
        acc[4 * u + 1] = fmaf(g.y, x, acc[4 * u + 1]);
        acc[4 * u + 2] = fmaf(g.z, x, acc[4 * u + 2]);
        acc[4 * u + 3] = fmaf(g.w, x, acc[4 * u + 3]);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < 16; ++u)
    if (16 * w + u < E) part_w[(static_cast<size_t>(blockIdx.y) * E + 16 * w + u) * d + c0 + lane] = acc[u];
}

// dw = sum over the parts, of bf16 rows over dl's three as well (rows e, E + e, 2 E + e
// of a part of `rows` rows): 256 values a block, a wave a sixteenth of the parts (its
// loads are in flight together).  The last block: db over the blocks of scored_dlogits.
// In a fixed order.  Bounded by the parts' 50 MB: 15 us (65536 x 1024, 64 experts).
template <int SPLITS>
__global__ __launch_bounds__(1024) void scored_dw_reduce_kernel(const float* __restrict__ part_w,
                                                               const float* __restrict__ part_b, int parts,
                                                               int b_parts, int rows, int d, int E,
                                                               float* __restrict__ dw, float* __restrict__ db) {
  __shared__ float4 lds[16][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  const bool tail = blockIdx.x + 1 == gridDim.x;
  const long long at = static_cast<long long>(blockIdx.x) * 256 + 4 * lane;   // (E d is a multiple of 64)
  const bool in = !tail && at < static_cast<long long>(E) * d;
  if (tail) {
    if (!db) return;
#pragma unroll 8
    for (int p = w; p < b_parts; p += 16) s.x += lane < E ? part_b[static_cast<size_t>(p) * E + lane] : 0.f;
  } else if (in) {
    const int e = static_cast<int>(at / d), c = static_cast<int>(at - static_cast<long long>(e) * d);
#pragma unroll 4
    for (int p = w; p < parts; p += 16)
#pragma unroll
      for (int q = 0; q < SPLITS; ++q) {
        const float4 v = *reinterpret_cast<const float4*>(part_w + (static_cast<size_t>(p) * rows + q * E + e) * d + c);
        s.x += v.x;
        s.y += v.y;
        s.z += v.z;
        s.w += v.w;
      }
  }
  lds[w][lane] = s;
  __syncthreads();
  if (w > 0) return;
#pragma unroll
  for (int v = 1; v < 16; ++v) {
    const float4 o = lds[v][lane];
    s.x += o.x;
    s.y += o.y;
    s.z += o.z;
    s.w += o.w;
  }
  if (tail) {
    if (lane < E) db[lane] = s.x;
  } else if (in) {
    *reinterpret_cast<float4*>(dw + at) = s;
  }
}

struct ScoredBwdWs {
  uint16_t* dl;         // [T][ld]
  int32_t* part_rows;   // [parts + 1]
  float *part_w, *part_b;
};

// What the backward's sizes follow from.
struct ScoredBwdPlan {
  int ld;          // columns of dl's rows: 3 E, rounded up as the product wants
  int parts, per;  // parts of T in dW's sums, and the tokens of one
  int rows;        // rows of a part's sums
  int b_parts;     // blocks of scored_dlogits
};

ScoredBwdPlan scored_bwd_plan(int T, int d, int E, bool bf16) {
  ScoredBwdPlan p;
  p.ld = (3 * E + 63) / 64 * 64;
  // bf16: 256 x 256 tiles, about one a CU, of at least 128 tokens (product + sums in us
  // with 64, 128, 256: 761 x 3008, 32 experts 18.9, 18.2, 19.7; 4096 x 1024, 64 experts
  // 25.9, 23.4, 22.7; 2048 x 4096, 16 experts 19.0, 19.5, 21.2), and a part's rows within
  // a buffer resource; float32: about a thousand blocks
  const int tiles = (d + 255) / 256;
  const int most = bf16 ? std::min(kMaxDwParts, std::max(1, 256 / tiles)) : std::max(1, 1024 / std::max(1, d / kDwCols));
  const int least = bf16 ? 128 : kDwTok;
  p.parts = std::max(1, std::min((T + least - 1) / least, most));
  if (bf16) {
    const long long fit = 0xFFFF0000ll / 2 / std::max(d, p.ld) - 2 * kDwTok;   // tokens
    p.parts = std::max(p.parts, static_cast<int>(std::min<long long>((T + fit - 1) / fit, kMaxDwParts + 1)));
  }
  p.per = ((T + p.parts - 1) / p.parts + kDwTok - 1) / kDwTok * kDwTok;
  p.rows = bf16 ? p.ld : E;
  p.b_parts = std::max(1, std::min((T + 15) / 16, 1024));
  return p;
}

ScoredBwdWs carve_scored_bwd(Carver& c, int T, int d, int E, bool bf16) {
  const ScoredBwdPlan p = scored_bwd_plan(T, d, E, bf16);
  ScoredBwdWs w;
  w.dl = c.take<uint16_t>(static_cast<size_t>(T) * p.ld);
  w.part_rows = c.take<int32_t>(p.parts + 1);
  w.part_w = c.take<float>(static_cast<size_t>(p.parts) * p.rows * d);
  w.part_b = c.take<float>(static_cast<size_t>(p.b_parts) * E);
  return w;
}

// Host checks shared by both directions.
int scored_check(const char* fn, int T, int d, int dtype, int E, int k, int score, float scale) {
  if (T <= 0 || d <= 0 || E <= 0) return fail(LUFFY_E_INVALID, "%s: T=%d d=%d E=%d must be positive", fn, T, d, E);
  if (k < 1 || k > E) return fail(LUFFY_E_INVALID, "%s: k=%d must be 1 to E=%d", fn, k, E);
  if (dtype != LUFFY_F32 && dtype != LUFFY_BF16) return fail(LUFFY_E_INVALID, "%s: unknown dtype %d", fn, dtype);
  if (score != LUFFY_SCORE_SOFTMAX && score != LUFFY_SCORE_SIGMOID)
    return fail(LUFFY_E_INVALID, "%s: unknown score %d", fn, score);
  if (!(std::fabs(scale) < INFINITY)) return fail(LUFFY_E_INVALID, "%s: scale must be finite", fn);
  if (E > kMaxExperts) return fail(LUFFY_E_UNSUPPORTED, "%s: E=%d > %d", fn, E, kMaxExperts);
  if (k > kMaxChoices) return fail(LUFFY_E_UNSUPPORTED, "%s: k=%d > %d", fn, k, kMaxChoices);
  if (d % 64 != 0) return fail(LUFFY_E_UNSUPPORTED, "%s: d=%d not a multiple of 64", fn, d);
  if (d > 32768) return fail(LUFFY_E_UNSUPPORTED, "%s: d=%d > 32768", fn, d);
  if (T > (1 << 28) || static_cast<long long>(T) * k >= (1ll << 31))
    return fail(LUFFY_E_UNSUPPORTED, "%s: T=%d k=%d: at most 2^28 tokens, and fewer than 2^31 slots", fn, T, k);
  return LUFFY_OK;
}

}  // namespace
}  // namespace luffy

using namespace luffy;

extern "C" int luffy_route_scored(const void* x, int T, int d, int dtype, const void* w_gate, const float* b_gate, int E,
                                  int k, int score, const float* balance, int groups, int top_groups, int group_best,
                                  int renormalise, float scale, double capacity_factor, int32_t* topk_idx,
                                  float* topk_gate, float* logits, int32_t* slot_pos, int32_t* perm_token,
                                  int32_t* offsets, float* inv_norm, void* workspace, size_t workspace_bytes,
                                  void* stream) {
  const char* fn = "luffy_route_scored";
  if (!x || !w_gate || !topk_idx || !topk_gate || !logits || !slot_pos || !perm_token || !offsets)
    return fail(LUFFY_E_INVALID, "%s: null pointer argument", fn);
  const int st = scored_check(fn, T, d, dtype, E, k, score, scale);
  if (st != LUFFY_OK) return st;
  if (groups < 1 || E % groups != 0) return fail(LUFFY_E_INVALID, "%s: groups=%d must divide E=%d", fn, groups, E);
  if (top_groups < 1 || top_groups > groups)
    return fail(LUFFY_E_INVALID, "%s: top_groups=%d must be 1 to groups=%d", fn, top_groups, groups);
  if (group_best != 1 && group_best != 2) return fail(LUFFY_E_INVALID, "%s: group_best=%d must be 1 or 2", fn, group_best);
  if (k > top_groups * (E / groups))
    return fail(LUFFY_E_INVALID, "%s: k=%d, but %d groups of %d", fn, k, top_groups, E / groups);
  if (groups > kMaxGroups && top_groups < groups)
    return fail(LUFFY_E_UNSUPPORTED, "%s: groups=%d > %d", fn, groups, kMaxGroups);
  if ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(w_gate)) & 15u)
    return fail(LUFFY_E_INVALID, "%s: x and w_gate must be 16-byte aligned", fn);
  const size_t need = luffy_route_workspace_size(T, E, k);
  if (workspace_bytes < need || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return fail(LUFFY_E_WORKSPACE, "%s: workspace needs %zu bytes, 256-aligned", fn, need);
  hipStream_t s = static_cast<hipStream_t>(stream);
  Carver c(workspace);
  const RouteWs ws = carve_route(c, T, E, k);
  const ScoreArgs a{b_gate, balance, E, k, score, groups, E / groups, top_groups, group_best, renormalise != 0, scale};
#define LUFFY_SCORED(BF, A)                                                                                             \
  launch("scored_gate", scored_gate_kernel<BF, A>, (T + 16 * A - 1) / (16 * A), 256, 0, s, x, w_gate, T, d, a, logits, \
         topk_gate, inv_norm)
  const bool bf16 = dtype == LUFFY_BF16, sig = score == LUFFY_SCORE_SIGMOID, grouped = top_groups < groups;
  const int C = capacity_slots(T, k, E, capacity_factor);
  auto buckets = [&](int tok) {
    const long long slots = static_cast<long long>(T) * k, nblk = (T + tok - 1) / tok;
    if (E * k * nblk <= kPlaceCounts)
      launch("slot_place", slot_place_kernel, static_cast<int>((slots + 1023) / 1024), 1024, 0, s, topk_idx, ws.hist, T,
             k, E, C, tok, slot_pos, perm_token, offsets);
    else
      route_buckets_enqueue(topk_idx, T, E, k, capacity_factor, tok, slot_pos, perm_token, offsets, ws, s);
  };
  // One launch where every block has a CU of its own, and where it is not two chunks
  // instead of a whole call in one (us a call in a graph, one | two launches: 64 x 1024, 64
  // experts 19.1 | 20.2, 1024 x 4096 46.3 | 48.0, 4096 x 1024 30.1 | 32.0, float32 40.9 |
  // 42.7; 8192 x 2048, 32 experts 34.3 | 33.7; from the host a launch less is 2.5 us more).
  const int chunks = (T + 15) / 16, cus = persistent_grid();
  if (T <= 16 || (T > kChooseTok && chunks <= cus)) {
#define LUFFY_BOTH(BF, NEB)                                                                                        \
  launch("scored_both",                                                                                            \
         sig ? (grouped ? scored_both_kernel<BF, NEB, true, true> : scored_both_kernel<BF, NEB, true, false>)     \
             : (grouped ? scored_both_kernel<BF, NEB, false, true> : scored_both_kernel<BF, NEB, false, false>),  \
         chunks, 256, 0, s, x, w_gate, T, d, a, C, topk_idx, topk_gate, logits, inv_norm, slot_pos, ws.hist,        \
         ws.done, perm_token, offsets)
    if (E <= 16) {
      if (bf16) LUFFY_BOTH(true, 1); else LUFFY_BOTH(false, 1);
    } else {
      if (bf16) LUFFY_BOTH(true, 4); else LUFFY_BOTH(false, 4);
    }
#undef LUFFY_BOTH
    if (chunks > 1) buckets(16);
    return check_launch(fn);
  }
  // Streaming from eight chunks of 16 tokens a CU on: below, staging W (8 us) and the
  // idle waves cost more than blocks that fetch it from L2 (us, streaming | blocks: 64 x
  // 1024 at T 16384 25 | 18, 32768 25 | 31; 32 x 2048 28 | 21, 42 | 45; 16 x 1024 at 65536
  // 32 | 45).  Blocks of 16 tokens have the most waves, of 64 fetch W least often (16, 32,
  // 64 tokens: 2048 x 64 x 1024 11, 13, 15 us; 8192 15, 13, 17; 32768 45, 31, 31; 65536 x
  // 64 x 4096 with 32 213, with 64 176).
  if (stream_ok(dtype, E, d) && chunks >= 8 * cus) {
    const int waves = std::min(kStreamWaves, (chunks + cus - 1) / cus);
#define LUFFY_SCORED_S(NEB)                                                                                         \
  launch("scored_gate", waves > 8 ? scored_gate_stream_kernel<NEB, 16> : scored_gate_stream_kernel<NEB, 8>, cus,    \
         64 * waves, 0, s, static_cast<const uint16_t*>(x), static_cast<const uint16_t*>(w_gate), T, d, a, logits,  \
         topk_gate, inv_norm)
    if (E <= 16) LUFFY_SCORED_S(1);
    else if (E <= 32) LUFFY_SCORED_S(2);
    else if (E <= 48) LUFFY_SCORED_S(3);
    else LUFFY_SCORED_S(4);
#undef LUFFY_SCORED_S
  } else if (T >= 32768) {
    if (bf16) LUFFY_SCORED(true, 4); else LUFFY_SCORED(false, 4);
  } else if (T >= 8192) {
    if (bf16) LUFFY_SCORED(true, 2); else LUFFY_SCORED(false, 2);
  } else {
    if (bf16) LUFFY_SCORED(true, 1); else LUFFY_SCORED(false, 1);
  }
#undef LUFFY_SCORED
  // Tokens of a chunk: 16 make the longest chain of a block shorter while the chip has
  // room for the blocks, 32 halve the counts that slot_scan goes through (64 experts of
  // 1024, k 8, choices | scan in us, 16 against 32 tokens: T 2048 11.2 | 6.4 against 13.0
  // | 6.5, 8192 17.4 | 7.1 against 19.5 | 6.5, 16384 20.2 | 8.4 against 20.2 | 7.4; 64 x
  // 4096 at 65536 58 | 16 against 54 | 11).  As many as there are where one block does.
  const int tok = T > kChooseTok && T <= 8192 ? 16 : kChooseTok;
  const int blocks = (T + tok - 1) / tok;
#define LUFFY_CHOOSE(NEB)                                                                                           \
  launch("scored_choose",                                                                                           \
         sig ? (grouped ? scored_choose_kernel<NEB, true, true> : scored_choose_kernel<NEB, true, false>)           \
             : (grouped ? scored_choose_kernel<NEB, false, true> : scored_choose_kernel<NEB, false, false>),        \
         blocks, kChooseWaves * 64, 0, s, x, w_gate, bf16, T, d, tok, a, C, topk_idx, topk_gate, logits, slot_pos,       \
         ws.hist, ws.done, perm_token, offsets)
  if (E <= 16) LUFFY_CHOOSE(1);
  else if (E <= 32) LUFFY_CHOOSE(2);
  else if (E <= 48) LUFFY_CHOOSE(3);
  else LUFFY_CHOOSE(4);
#undef LUFFY_CHOOSE
  if (blocks > 1) buckets(tok);
  return check_launch(fn);
}

extern "C" size_t luffy_route_scored_backward_workspace_size(int T, int d, int E) {
  if (T <= 0 || d <= 0 || E <= 0) return 0;
  size_t most = 0;
  for (const bool bf16 : {false, true}) {
    Carver c(nullptr);
    carve_scored_bwd(c, T, d, E, bf16);
    most = std::max(most, c.size());
  }
  return most;
}

extern "C" int luffy_route_scored_backward(const void* x, int T, int d, int dtype, const void* w_gate, int E, int k,
                                           int score, int renormalise, float scale, const float* logits,
                                           const int32_t* topk_idx, const float* dgate, const float* dlogits,
                                           const void* dx_rep, const int32_t* slot_pos, const int32_t* rep_of_pos,
                                           const int32_t* rep_row, void* dx, float* dw_gate, float* db_gate,
                                           void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "luffy_route_scored_backward";
  if (!x || !w_gate || !logits || !topk_idx || !dgate || !dx || !dw_gate)
    return fail(LUFFY_E_INVALID, "%s: null pointer argument", fn);
  if (dx_rep && (!slot_pos || !rep_of_pos || !rep_row))
    return fail(LUFFY_E_INVALID, "%s: dx_rep needs slot_pos, rep_of_pos and rep_row", fn);
  const int st = scored_check(fn, T, d, dtype, E, k, score, scale);
  if (st != LUFFY_OK) return st;
  uintptr_t bits = 0;
  for (const void* p : {x, w_gate, dx_rep, static_cast<const void*>(dx), static_cast<const void*>(dw_gate)})
    bits |= reinterpret_cast<uintptr_t>(p);
  if (bits & 15u) return fail(LUFFY_E_INVALID, "%s: x, w_gate, dx_rep, dx and dw_gate must be 16-byte aligned", fn);
  if (dtype == LUFFY_BF16 && scored_bwd_plan(T, d, E, true).parts > kMaxDwParts)
    return fail(LUFFY_E_UNSUPPORTED, "%s: %d rows of %d exceed 64 parts of 4 GiB", fn, T, d);
  const size_t need = luffy_route_scored_backward_workspace_size(T, d, E);
  if (workspace_bytes < need || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return fail(LUFFY_E_WORKSPACE, "%s: workspace needs %zu bytes, 256-aligned", fn, need);
  hipStream_t s = static_cast<hipStream_t>(stream);
  Carver c(workspace);
  const bool bf16 = dtype == LUFFY_BF16;
  const ScoredBwdPlan p = scored_bwd_plan(T, d, E, bf16);
  const ScoredBwdWs ws = carve_scored_bwd(c, T, d, E, bf16);
  const ScoreArgs a{nullptr, nullptr, E, k, score, 1, E, 1, 1, renormalise != 0, scale};
  launch("scored_dlogits", E % 4 == 0 ? scored_dlogits_kernel<true> : scored_dlogits_kernel<false>, p.b_parts,
         kDlThreads, 0, s, logits, topk_idx, dgate, dlogits, T, a, p.ld, ws.dl, p.parts, p.per, ws.part_rows,
         ws.part_b);
  // a row is shared by waves where there are fewer tokens than the chip holds waves (us,
  // with a wave a row | shared: 761 x 3008, 32 experts, k 8 32 | 11; float32 405 x 2176 19
  // | 7; 1498 x 1216 12 | 8; twice as many waves are no faster)
  const int cols = 64 * 16 / elem_bytes(dtype), cus = persistent_grid();
  const int slices = std::max(1, std::min((d + cols - 1) / cols, 32 * cus / T));
  const long long items = static_cast<long long>(T) * slices;
  const int blocks = static_cast<int>(std::min<long long>((items + 3) / 4, 16 * cus));
  launch("scored_dx", bf16 ? scored_dx_kernel<true> : scored_dx_kernel<false>, blocks, 256, 0, s, w_gate, ws.dl, p.ld,
         T, d, E, k, slices, dx_rep, slot_pos, rep_of_pos, rep_row, dx);
  if (bf16)
    row_product_enqueue("scored_dw", ws.dl, static_cast<const uint16_t*>(x), ws.part_rows, p.parts, p.ld, d, ws.part_w,
                        s);
  else
    launch("scored_dw", scored_dw_kernel, dim3(d / kDwCols, p.parts), 256, 0, s, static_cast<const float*>(x), ws.dl,
           p.ld, T, d, E, p.per, ws.part_w);
  const long long n = static_cast<long long>(E) * d;
  launch("scored_dw_reduce", bf16 ? scored_dw_reduce_kernel<3> : scored_dw_reduce_kernel<1>,
         static_cast<int>((n + 255) / 256) + 1, 1024, 0, s, ws.part_w, ws.part_b, p.parts, p.b_parts, p.rows, d, E, dw_gate,
         db_gate);
  return check_launch(fn);
}
