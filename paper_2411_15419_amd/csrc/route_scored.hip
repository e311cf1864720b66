// luffy_route_scored and luffy_route_scored_backward: a router with softmax or
// sigmoid scores, a bias for balance, groups of experts and up to eight experts a
// token.
//
// Forward kernels:
//   scored_gate    logits on MFMA (float32 sums), scores and a first choice; a token
//                  with a deciding gap within the sums' error bound is marked (its
//                  experts stored as -1 - e)
//   scored_settle  decides the marked tokens in float64 from exact products, ranks
//                  every slot among its chunk's slots of the same expert, and leaves
//                  the chunks' counts
//   slot_scan, slot_scatter  (route.hip) bucket offsets and positions
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "luffy_common.h"
#include "route.h"

namespace luffy {
namespace {

constexpr int kMaxChoices = 8, kMaxGroups = 16;
constexpr int kSettleTok = 64;   // tokens of a scored_settle block and histogram chunk
constexpr float kLog2e = 1.44269504088896341f;

struct ScoreArgs {
  const float *bias, *balance;   // [E] or null
  int E, k, score, groups, group_size, top_groups, best, renormalise;
  float scale;
};

template <int N>
__device__ __forceinline__ uint32_t ror16(uint32_t x) {   // by N lanes inside each row of 16
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x120 + N, 0xF, 0xF, false));
}
template <int N>
__device__ __forceinline__ float ror16f(float x) { return __uint_as_float(ror16<N>(__float_as_uint(x))); }
// Every lane of a row of 16 ends with the row's maximum or sum.
__device__ __forceinline__ uint32_t max16(uint32_t x) {
  x = max(x, ror16<8>(x));
  x = max(x, ror16<4>(x));
  x = max(x, ror16<2>(x));
  return max(x, ror16<1>(x));
}
__device__ __forceinline__ float max16f(float x) {
  x = fmaxf(x, ror16f<8>(x));
  x = fmaxf(x, ror16f<4>(x));
  x = fmaxf(x, ror16f<2>(x));
  return fmaxf(x, ror16f<1>(x));
}
__device__ __forceinline__ float sum16(float x) {
  x += ror16f<8>(x);
  x += ror16f<4>(x);
  x += ror16f<2>(x);
  return x + ror16f<1>(x);
}
// The two largest of a row, a >= b in every lane.
__device__ __forceinline__ void best2_16(float& a, float& b) {
  auto merge = [&](float c, float e) {
    b = fmaxf(fminf(a, c), fmaxf(b, e));
    a = fmaxf(a, c);
  };
  merge(ror16f<8>(a), ror16f<8>(b));
  merge(ror16f<4>(a), ror16f<4>(b));
  merge(ror16f<2>(a), ror16f<2>(b));
  merge(ror16f<1>(a), ror16f<1>(b));
}

// Order-preserving key of a value with its expert in the low six bits: among
// values equal in their top 26 bits the lower expert has the larger key.  What is
// dropped is less than 2^-17 of the value.
__device__ __forceinline__ uint32_t choice_key(float v, int e) {
  const uint32_t u = __float_as_uint(v);
  const uint32_t o = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  return (o & ~63u) | static_cast<uint32_t>(63 - e);
}
__device__ __forceinline__ float key_value(uint32_t key) {
  if (key == 0u) return -INFINITY;   // no expert
  const uint32_t o = key & ~63u;
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o);
}

// Whether a > b in truth, each known to `rel` of itself and `abs` besides.  A b of
// -infinity (an expert that is masked out) is below every other a, unless abs says
// that the numbers left float32's range.
__device__ __forceinline__ bool apart(float a, float b, float rel, float abs) {
  if (b == -INFINITY && a > -INFINITY) return abs < INFINITY;
  return a - b > fmaf(rel, fabsf(a) + fabsf(b), 2.0f * abs);
}

// 1 / (1 + e^-l) times e^-shift, shift <= 0: no overflow for any l.
__device__ __forceinline__ float sigmoid_shifted(float l, float shift) {
  return __builtin_amdgcn_exp2f((fminf(l, 0.f) - shift) * kLog2e) /
         (1.0f + __builtin_amdgcn_exp2f(-fabsf(l) * kLog2e));
}

// Choice of one token by the 16 lanes of a row, lane m with the logits l[j] of
// experts 16 j + m (those past E are ignored).  dl bounds the logits' error.  Lane
// i < k ends with the i-th expert and its gate; `marked` is set for the row where a
// deciding gap may be of either sign:
//   logits         2 dl
//   sigmoid + bias a score moves by at most dl / 4, its evaluation and the sum by
//                  less than 2^-20 (1 + |c|)
//   softmax + bias by at most 2 dl of itself (its own exponential and the sum of
//                  all), evaluation as above
// and 2^-17 of either value for the keys; the sum of a group's two best moves by
// twice that.
template <int NEB>
__device__ __forceinline__ void choose16(const float (&l)[NEB], const float (&bal)[NEB], const int (&grp)[NEB],
                                         const ScoreArgs& a, float dl, int& expert, float& gate, bool& marked) {
  const int lane = threadIdx.x & 63, m = lane & 15, row = lane & 48;
  const bool sig = a.score == LUFFY_SCORE_SIGMOID, biased = a.balance != nullptr;
  const bool grouped = a.top_groups < a.groups;
  float top = -INFINITY, inv_z = 0.f;
  if (!sig) {
    float z = 0.f;
#pragma unroll
    for (int j = 0; j < NEB; ++j) top = fmaxf(top, 16 * j + m < a.E ? l[j] : -INFINITY);
    top = max16f(top);
#pragma unroll
    for (int j = 0; j < NEB; ++j)
      z += 16 * j + m < a.E ? __builtin_amdgcn_exp2f((l[j] - top) * kLog2e) : 0.f;
    inv_z = 1.0f / sum16(z);
  }
  auto score = [&](float v) {
    return sig ? sigmoid_shifted(v, 0.f) : __builtin_amdgcn_exp2f((v - top) * kLog2e) * inv_z;
  };
  const float ds = sig ? 0.25f * dl + 0x1p-21f : fmaf(2.0f * inv_z, dl, 0x1p-21f);   // (inv_z: the largest score)
  float c[NEB];
#pragma unroll
  for (int j = 0; j < NEB; ++j) {
    c[j] = biased ? score(l[j]) + bal[j] : l[j];
    if (c[j] != c[j]) c[j] = -INFINITY;   // no number: chosen last
  }
  const float dc = biased ? ds : dl;
  marked = false;
  uint32_t kept = ~0u;   // groups
  if (grouped) {
    const bool by_score = !biased && a.best == 2;
    const float dg = (a.best == 2 ? 2.0f : 1.0f) * (by_score ? ds : dc);
    float value = -INFINITY;   // lane g: group g's
    for (int g = 0; g < a.groups; ++g) {
      float b1 = -INFINITY, b2 = -INFINITY;
#pragma unroll
      for (int j = 0; j < NEB; ++j) {
        float v = by_score ? score(l[j]) : c[j];
        if (!(v == v) || grp[j] != g || 16 * j + m >= a.E) v = -INFINITY;
        b2 = fmaxf(b2, fminf(b1, v));
        b1 = fmaxf(b1, v);
      }
      best2_16(b1, b2);
      if (m == g) value = a.best == 2 && a.group_size > 1 ? b1 + b2 : b1;
    }
    bool open = m < a.groups;
    float last = 0.f;
    kept = 0;
    for (int r = 0; r < a.top_groups; ++r) {
      last = max16f(open ? value : -INFINITY);
      const uint32_t at = static_cast<uint32_t>(__ballot(open && value == last) >> row) & 0xFFFFu;
      const int g = __ffs(static_cast<int>(at)) - 1;
      kept |= 1u << g;
      if (m == g) open = false;
    }
    const float next = max16f(open ? value : -INFINITY);
    marked = !apart(last, next, 0x1p-21f, dg);
  }
  uint32_t key[NEB];
#pragma unroll
  for (int j = 0; j < NEB; ++j) {
    const int e = 16 * j + m;
    key[j] = e < a.E && ((kept >> grp[j]) & 1u) ? choice_key(c[j], e) : 0u;
  }
  uint32_t bound = ~0u;
  float before = 0.f;
  expert = 0;
  for (int i = 0; i <= a.k; ++i) {
    uint32_t best = 0;
#pragma unroll
    for (int j = 0; j < NEB; ++j) best = max(best, key[j] < bound ? key[j] : 0u);
    best = max16(best);
    const float v = key_value(best);
    if (i > 0 && best != 0u) marked = marked || !apart(before, v, 0x1p-17f, dc);
    if (i < a.k && m == i) expert = 63 - static_cast<int>(best & 63u);
    bound = best;
    before = v;
  }
  // gates, from the chosen experts' logits
  float own = 0.f;
#pragma unroll
  for (int j = 0; j < NEB; ++j) {
    const float v = __shfl(l[j], row | (expert & 15), 64);
    if ((expert >> 4) == j) own = v;
  }
  const bool mine = m < a.k;
  if (a.renormalise) {
    const float most = max16f(mine ? own : -INFINITY);
    const float s = !mine ? 0.f
                          : sig ? sigmoid_shifted(own, fminf(most, 0.f))
                                : __builtin_amdgcn_exp2f((own - most) * kLog2e);
    gate = a.scale * (s / sum16(s));
  } else {
    gate = a.scale * score(own);
  }
}

// Logits of TOK = 16 A tokens a block: four waves, each a quarter of d, on 16-token
// by 16-expert MFMA tiles, two batches of two K steps in flight; the quarters are
// added in LDS.  The rows' and the experts' squared norms come from the same
// fragments (the diagonals of their own Grams): with n MFMA sums in a row and their
// few joins the error of a logit is at most (n + 16) 2^-24 |x| |w| (every rounding
// is relative to the absolute sum of the products, which is at most |x| |w|), the
// norms being a little off covered by a factor of 1.01.
template <bool BF16, int A>
__global__ __launch_bounds__(256) void scored_gate_kernel(const void* __restrict__ xv, const void* __restrict__ wv,
                                                          int T, int d, ScoreArgs a, int32_t* __restrict__ topk_idx,
                                                          float* __restrict__ topk_gate, float* __restrict__ logits,
                                                          float* __restrict__ inv_norm) {
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
    f32x4 acc[A][4], sqx[A], sqw[4];
    const Elem *xrow[A], *wrow[4];
#pragma unroll
    for (int i = 0; i < A; ++i) {
      sqx[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      xrow[i] = X + static_cast<size_t>(min(t0 + 16 * i + m, T - 1)) * d + VL * q;
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      sqw[j] = f32x4{0.f, 0.f, 0.f, 0.f};
      wrow[j] = W + static_cast<size_t>(min(16 * j + m, E - 1)) * d + VL * q;
    }
    constexpr int B = 2;
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
    auto compute = [&](const Pack16 (&x)[B][A], const Pack16 (&ww)[B][4]) {
#pragma unroll
      for (int u = 0; u < B; ++u) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (j >= neb) break;
          sqw[j] = mma(ww[u][j], ww[u][j], sqw[j]);
#pragma unroll
          for (int i = 0; i < A; ++i) acc[i][j] = mma(x[u][i], ww[u][j], acc[i][j]);
        }
#pragma unroll
        for (int i = 0; i < A; ++i) sqx[i] = mma(x[u][i], x[u][i], sqx[i]);
      }
    };
    if (s_lo < s_hi) load(s_lo, xa[0], wa[0]);
    for (int s0 = s_lo; s0 < s_hi; s0 += 2 * B) {
      if (s0 + B < s_hi) load(s0 + B, xa[1], wa[1]);
      compute(xa[0], wa[0]);
      if (s0 + B >= s_hi) break;
      if (s0 + 2 * B < s_hi) load(s0 + 2 * B, xa[0], wa[0]);
      compute(xa[1], wa[1]);
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
        if (j < neb) *reinterpret_cast<f32x4*>(&part[w][16 * j + m][16 * i + 4 * q]) = acc[i][j];
  }
  __syncthreads();
  float bias[4], bal[4], wmost = 0.f;
  int grp[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int e = 16 * j + m;
    const bool in = e < E;
    bias[j] = in && a.bias ? a.bias[e] : 0.f;
    bal[j] = in && a.balance ? a.balance[e] : 0.f;
    grp[j] = in && a.top_groups < a.groups ? e / a.group_size : 0;
    const float sq = in ? ((wsq[0][e] + wsq[1][e]) + wsq[2][e]) + wsq[3][e] : 0.f;
    wmost = sq > wmost || sq != sq ? sq : wmost;   // NaN stays
  }
  // (a NaN norm marks every token: fmaxf would drop it)
  wmost = __any(wmost != wmost) ? NAN : max16f(wmost);
  for (int it = w; it < TOK / 4; it += 4) {
    const int tl = 4 * it + q, t = t0 + tl;
    const float ss = ((xsq[0][tl] + xsq[1][tl]) + xsq[2][tl]) + xsq[3][tl];
    const float dl = 1.01f * static_cast<float>(per * (BF16 ? 1 : 4) + 16) * 0x1p-24f * sqrtf(ss) * sqrtf(wmost);
    float l[4], most = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int e = min(16 * j + m, E - 1);
      l[j] = ((part[0][e][tl] + part[1][e][tl]) + part[2][e][tl]) + part[3][e][tl] + bias[j];
      most = fmaxf(most, fabsf(bias[j]));
    }
    int expert;
    float gate;
    bool marked;
    choose16(l, bal, grp, a, fmaf(0x1p-23f, max16f(most), dl), expert, gate, marked);
    if (t >= T) continue;
    if (logits) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (16 * j + m < E) logits[static_cast<size_t>(t) * E + 16 * j + m] = l[j];
    }
    if (m < a.k) {
      topk_idx[static_cast<size_t>(t) * a.k + m] = marked ? -1 - expert : expert;
      topk_gate[static_cast<size_t>(t) * a.k + m] = gate;
    }
    if (inv_norm && m == 0) inv_norm[t] = ss > 0.f ? 1.0f / sqrtf(ss) : 0.f;
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

// A block's kSettleTok tokens: the marked ones are decided from float64 logits of
// exact products (the waves share the experts, then wave 0 has one a lane), and
// waves rank the slots of a choice each.
template <bool BF16>
__global__ __launch_bounds__(256) void scored_settle_kernel(const void* __restrict__ xv, const void* __restrict__ wv,
                                                            int T, int d, ScoreArgs a, int32_t* __restrict__ topk_idx,
                                                            float* __restrict__ topk_gate, float* __restrict__ logits,
                                                            int32_t* __restrict__ slot_rank,
                                                            int32_t* __restrict__ hist, int* __restrict__ scan_done) {
  using Elem = std::conditional_t<BF16, uint16_t, float>;
  constexpr int VL = 16 / sizeof(Elem);
  __shared__ int choice[kMaxChoices][kSettleTok];
  __shared__ double lg[kMaxExperts], val[kMaxExperts], gval[kMaxGroups];
  __shared__ int cnt[4][kMaxExperts];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int ch = blockIdx.x, t0 = ch * kSettleTok, E = a.E, k = a.k, nch = gridDim.x;
  if (ch == 0 && threadIdx.x == 0) *scan_done = 0;   // armed for slot_scan
  for (int i = threadIdx.x; i < kSettleTok * k; i += 256) {
    const int tl = i / k, j = i - tl * k;
    choice[j][tl] = t0 + tl < T ? topk_idx[static_cast<size_t>(t0) * k + i] : 0;
  }
  __syncthreads();
  uint64_t open = __ballot(choice[0][lane] < 0);   // the same in every wave
  while (open) {
    const int tl = __ffsll(static_cast<long long>(open)) - 1;
    open &= open - 1;
    const size_t t = t0 + tl;
    const Elem* x = static_cast<const Elem*>(xv) + t * d;
    for (int e = w; e < E; e += 4) {
      const Elem* we = static_cast<const Elem*>(wv) + static_cast<size_t>(e) * d;
      double s = 0.0;
      for (int c = lane * VL; c < d; c += 64 * VL) {
        Pack16 xa, wa;
        xa.u4 = *reinterpret_cast<const uint4*>(x + c);
        wa.u4 = *reinterpret_cast<const uint4*>(we + c);
#pragma unroll
        for (int u = 0; u < VL; ++u) {
          if constexpr (BF16)
            s = fma(static_cast<double>(bf16_to_f32(xa.h[u])), static_cast<double>(bf16_to_f32(wa.h[u])), s);
          else
            s = fma(static_cast<double>(xa.f[u]), static_cast<double>(wa.f[u]), s);
        }
      }
      s = wave_sum64(s);
      if (lane == 0) lg[e] = s + (a.bias ? static_cast<double>(a.bias[e]) : 0.0);
    }
    __syncthreads();
    if (w == 0) {
      const bool in = lane < E, sig = a.score == LUFFY_SCORE_SIGMOID;
      const double l = in ? lg[lane] : -INFINITY;
      double s;
      if (sig) {
        s = 1.0 / (1.0 + exp(-l));
      } else {
        const double top = wave_max64(l), p = in ? exp(l - top) : 0.0;
        s = p / wave_sum64(p);
      }
      double c = a.balance ? s + (in ? static_cast<double>(a.balance[lane]) : 0.0) : l;
      if (!(c == c) || !in) c = -INFINITY;
      bool allowed = in;
      if (a.top_groups < a.groups) {
        val[lane] = !a.balance && a.best == 2 ? (s == s && in ? s : -INFINITY) : c;
        __builtin_amdgcn_wave_barrier();
        double g = -INFINITY;
        if (lane < a.groups) {
          double b1 = -INFINITY, b2 = -INFINITY;
          for (int u = 0; u < a.group_size; ++u) {
            const double v = val[lane * a.group_size + u];
            b2 = fmax(b2, fmin(b1, v));
            b1 = fmax(b1, v);
          }
          g = a.best == 2 && a.group_size > 1 ? b1 + b2 : b1;
          gval[lane] = g;
        }
        __builtin_amdgcn_wave_barrier();
        int rank = kMaxGroups;
        if (lane < a.groups) {
          rank = 0;
          for (int h = 0; h < a.groups; ++h) rank += gval[h] > g || (gval[h] == g && h < lane);
        }
        const uint64_t kept = __ballot(rank < a.top_groups);
        allowed = in && ((kept >> (in ? lane / a.group_size : 0)) & 1ull);
      }
      __builtin_amdgcn_wave_barrier();
      val[lane] = c;
      const uint64_t may = __ballot(allowed);
      __builtin_amdgcn_wave_barrier();
      int rank = 0;
      for (int e = 0; e < E; ++e)
        rank += ((may >> e) & 1ull) && (val[e] > c || (val[e] == c && e < lane));
      const bool chosen = allowed && rank < k;
      double gate = s;
      if (a.renormalise) {
        const double most = wave_max64(chosen ? l : -INFINITY);
        const double shift = sig ? fmin(most, 0.0) : most;
        const double p = !chosen ? 0.0 : sig ? exp(fmin(l, 0.0) - shift) / (1.0 + exp(-fabs(l))) : exp(l - shift);
        gate = p / wave_sum64(p);
      }
      if (chosen) {
        choice[rank][tl] = lane;
        topk_idx[t * k + rank] = lane;
        topk_gate[t * k + rank] = static_cast<float>(static_cast<double>(a.scale) * gate);
      }
      if (logits && in) logits[t * E + lane] = static_cast<float>(l);
    }
    __syncthreads();
  }
  // stable ranks among the chunk's slots of the same expert: the lanes that hold
  // it, by ballots on its bits
  const bool valid = t0 + lane < T;
  for (int j = w; j < k; j += 4) {
    const int e = choice[j][lane];
    const int key = valid ? e : 127;
    uint64_t same = ~0ull;
#pragma unroll
    for (int b = 0; b < 7; ++b) {
      const bool bit = (key >> b) & 1;
      const uint64_t bb = __ballot(bit);
      same &= bit ? bb : ~bb;
    }
    const int rank = __popcll(same & lanemask_lt());
    cnt[w][lane] = 0;
    __builtin_amdgcn_wave_barrier();
    if (valid && rank == 0) cnt[w][e] = __popcll(same);
    __builtin_amdgcn_wave_barrier();
    if (lane < E) hist[static_cast<size_t>(lane) * k * nch + static_cast<size_t>(j) * nch + ch] = cnt[w][lane];
    if (valid) slot_rank[static_cast<size_t>(t0 + lane) * k + j] = rank;
    __builtin_amdgcn_wave_barrier();
  }
}

// ---------------------------------------------------------------- backward
// dl, the logits' gradient: with r_j = s_j / sum of the chosen (shifted as in the
// forward, so that nothing under- or overflows)
//   renormalised       dl_j = scale r_j (dg_j - sum_i dg_i r_i), times 1 - s_j for
//                      sigmoid scores; 0 for experts not chosen
//   sigmoid            dl_j = scale dg_j s_j (1 - s_j)
//   softmax            dl_e = s_e (ds_e - sum_i ds_i s_i), ds_j = scale dg_j
// plus what the caller adds.  A wave a token, an expert a lane.
__global__ __launch_bounds__(256) void scored_dlogits_kernel(const float* __restrict__ logits,
                                                             const int32_t* __restrict__ topk_idx,
                                                             const float* __restrict__ dgate,
                                                             const float* __restrict__ extra, int T, ScoreArgs a,
                                                             float* __restrict__ dl) {
  const int lane = threadIdx.x & 63, E = a.E, k = a.k;
  const bool sig = a.score == LUFFY_SCORE_SIGMOID, in = lane < E;
  for (long long t = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 6); t < T;
       t += static_cast<long long>(gridDim.x) * 4) {
    const float l = in ? logits[t * E + lane] : -INFINITY;
    float dg = 0.f;   // of this lane's expert, 0 if it was not chosen
    bool chosen = false;
    for (int j = 0; j < k; ++j)
      if (topk_idx[t * k + j] == lane) {
        dg += dgate[t * k + j];
        chosen = true;
      }
    auto wave_sum = [](float v) {
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
      return v;
    };
    auto wave_max = [](float v) {
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
      return v;
    };
    float g;
    if (a.renormalise) {
      const float most = wave_max(chosen ? l : -INFINITY), shift = sig ? fminf(most, 0.f) : most;
      const float p = !chosen ? 0.f : sig ? expf(fminf(l, 0.f) - shift) / (1.0f + expf(-fabsf(l))) : expf(l - shift);
      const float r = p / wave_sum(p), mean = wave_sum(dg * r);
      g = chosen ? a.scale * r * (dg - mean) : 0.f;
      if (sig && chosen) g *= 1.0f / (1.0f + expf(l));
    } else if (sig) {
      const float e = expf(-fabsf(l));
      g = chosen ? a.scale * dg * e / ((1.0f + e) * (1.0f + e)) : 0.f;
    } else {
      const float top = wave_max(l);
      const float p = in ? expf(l - top) : 0.f;
      const float s = p / wave_sum(p), mean = wave_sum(dg * s);
      g = s * a.scale * (dg - mean);
    }
    if (in) dl[t * E + lane] = g + (extra ? extra[t * E + lane] : 0.f);
  }
}

// dx of a token a wave: its experts' rows of W by dl, and the representatives'
// rows of dx_rep that are this token's.
template <bool BF16>
__global__ __launch_bounds__(256) void scored_dx_kernel(const void* __restrict__ wv, const float* __restrict__ dl,
                                                        int T, int d, int E, int k, const void* __restrict__ dx_rep,
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
  for (long long t = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 6); t < T;
       t += static_cast<long long>(gridDim.x) * 4) {
    const float g = lane < E ? dl[t * E + lane] : 0.f;
    const uint64_t used = __ballot(g != 0.f);
    int row = -1;
    if (dx_rep && lane < k) {
      const int p = slot_pos[t * k + lane];
      if (p >= 0 && rep_of_pos[p] == p) row = rep_row[p];
    }
    for (int c = lane * VL; c < (d + 64 * VL - 1) / (64 * VL) * (64 * VL); c += 64 * VL) {
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

// Part of dW = dl^T x and db: 64 columns by the tokens of part blockIdx.y, every
// expert; 64 tokens at a time in LDS, 16 experts a wave, a column a lane.
template <bool BF16>
__global__ __launch_bounds__(256) void scored_dw_kernel(const void* __restrict__ xv, const float* __restrict__ dl,
                                                        int T, int d, int E, int per, float* __restrict__ part_w,
                                                        float* __restrict__ part_b) {
  using Elem = std::conditional_t<BF16, uint16_t, float>;
  constexpr int VL = 16 / sizeof(Elem);
  __shared__ __attribute__((aligned(16))) float xs[kDwTok][kDwCols], gs[kDwTok][kMaxExperts];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c0 = blockIdx.x * kDwCols;
  const int t_lo = blockIdx.y * per, t_hi = min(T, t_lo + per);
  float acc[16], db = 0.f;
#pragma unroll
  for (int u = 0; u < 16; ++u) acc[u] = 0.f;
  for (int t0 = t_lo; t0 < t_hi; t0 += kDwTok) {
    __syncthreads();
    for (int i = threadIdx.x; i < kDwTok * kDwCols / VL; i += 256) {
      const int tl = i / (kDwCols / VL), c = i % (kDwCols / VL) * VL;
      Pack16 v;
      v.u4 = make_uint4(0, 0, 0, 0);
      if (t0 + tl < t_hi)
        v.u4 = *reinterpret_cast<const uint4*>(static_cast<const Elem*>(xv) + static_cast<size_t>(t0 + tl) * d + c0 + c);
#pragma unroll
      for (int u = 0; u < VL; ++u) {
        if constexpr (BF16) xs[tl][c + u] = bf16_to_f32(v.h[u]);
        else xs[tl][c + u] = v.f[u];
      }
    }
    for (int i = threadIdx.x; i < kDwTok * kMaxExperts; i += 256) {
      const int tl = i / kMaxExperts, e = i % kMaxExperts;
      gs[tl][e] = t0 + tl < t_hi && e < E ? dl[static_cast<size_t>(t0 + tl) * E + e] : 0.f;
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
      if (w == 0) db += gs[tl][lane];
    }
  }
#pragma unroll
  for (int u = 0; u < 16; ++u)
    if (16 * w + u < E) part_w[(static_cast<size_t>(blockIdx.y) * E + 16 * w + u) * d + c0 + lane] = acc[u];
  if (blockIdx.x == 0 && w == 0 && lane < E) part_b[static_cast<size_t>(blockIdx.y) * E + lane] = db;
}

// out[i] = sum over parts, in order.
__global__ __launch_bounds__(256) void scored_dw_reduce_kernel(const float* __restrict__ part_w,
                                                               const float* __restrict__ part_b, int parts,
                                                               long long n, int E, float* __restrict__ dw,
                                                               float* __restrict__ db) {
  const long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
  if (i < n) {
    float s = 0.f;
    for (int p = 0; p < parts; ++p) s += part_w[p * n + i];
    dw[i] = s;
  }
  if (db && i < E) {
    float s = 0.f;
    for (int p = 0; p < parts; ++p) s += part_b[static_cast<size_t>(p) * E + i];
    db[i] = s;
  }
}

struct ScoredBwdWs {
  float *dl, *part_w, *part_b;
};

// Parts of T in dW's sums: about a thousand blocks.
int dw_parts(int T, int d) {
  const int most = std::max(1, 1024 / std::max(1, d / kDwCols));
  return std::max(1, std::min((T + kDwTok - 1) / kDwTok, most));
}

ScoredBwdWs carve_scored_bwd(Carver& c, int T, int d, int E) {
  ScoredBwdWs w;
  const size_t parts = dw_parts(T, d);
  w.dl = c.take<float>(static_cast<size_t>(T) * E);
  w.part_w = c.take<float>(parts * E * d);
  w.part_b = c.take<float>(parts * E);
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
  if (static_cast<long long>(T) * k >= (1ll << 31)) return fail(LUFFY_E_UNSUPPORTED, "%s: T*k too large", fn);
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
  if (!x || !w_gate || !topk_idx || !topk_gate || !slot_pos || !perm_token || !offsets)
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
#define LUFFY_SCORED(BF, A)                                                                                         \
  launch("scored_gate", scored_gate_kernel<BF, A>, (T + 16 * A - 1) / (16 * A), 256, 0, s, x, w_gate, T, d, a, topk_idx, \
         topk_gate, logits, inv_norm)
  const bool bf16 = dtype == LUFFY_BF16;
  if (T >= 32768) { if (bf16) LUFFY_SCORED(true, 4); else LUFFY_SCORED(false, 4); }
  else if (T >= 8192) { if (bf16) LUFFY_SCORED(true, 2); else LUFFY_SCORED(false, 2); }
  else { if (bf16) LUFFY_SCORED(true, 1); else LUFFY_SCORED(false, 1); }
#undef LUFFY_SCORED
  launch("scored_settle", bf16 ? scored_settle_kernel<true> : scored_settle_kernel<false>,
         (T + kSettleTok - 1) / kSettleTok, 256, 0, s, x, w_gate, T, d, a, topk_idx, topk_gate, logits, slot_pos,
         ws.hist, ws.done);
  route_buckets_enqueue(topk_idx, T, E, k, capacity_factor, kSettleTok, slot_pos, perm_token, offsets, ws, s);
  return check_launch(fn);
}

extern "C" size_t luffy_route_scored_backward_workspace_size(int T, int d, int E) {
  if (T <= 0 || d <= 0 || E <= 0) return 0;
  Carver c(nullptr);
  carve_scored_bwd(c, T, d, E);
  return c.size();
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
  const size_t need = luffy_route_scored_backward_workspace_size(T, d, E);
  if (workspace_bytes < need || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return fail(LUFFY_E_WORKSPACE, "%s: workspace needs %zu bytes, 256-aligned", fn, need);
  hipStream_t s = static_cast<hipStream_t>(stream);
  Carver c(workspace);
  const ScoredBwdWs ws = carve_scored_bwd(c, T, d, E);
  const ScoreArgs a{nullptr, nullptr, E, k, score, 1, E, 1, 1, renormalise != 0, scale};
  const bool bf16 = dtype == LUFFY_BF16;
  const int waves = std::max(1, std::min((T + 3) / 4, 16 * persistent_grid()));
  const int parts = dw_parts(T, d), per = ((T + parts - 1) / parts + kDwTok - 1) / kDwTok * kDwTok;
  const long long n = static_cast<long long>(E) * d;
  launch("scored_dlogits", scored_dlogits_kernel, waves, 256, 0, s, logits, topk_idx, dgate, dlogits, T, a, ws.dl);
  launch("scored_dx", bf16 ? scored_dx_kernel<true> : scored_dx_kernel<false>, waves, 256, 0, s, w_gate, ws.dl, T, d, E,
         k, dx_rep, slot_pos, rep_of_pos, rep_row, dx);
  launch("scored_dw", bf16 ? scored_dw_kernel<true> : scored_dw_kernel<false>, dim3(d / kDwCols, parts), 256, 0, s, x,
         ws.dl, T, d, E, per, ws.part_w, ws.part_b);
  launch("scored_dw_reduce", scored_dw_reduce_kernel, static_cast<int>((n + 255) / 256), 256, 0, s, ws.part_w,
         ws.part_b, parts, n, E, dw_gate, db_gate);
  return check_launch(fn);
}
