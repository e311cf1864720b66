// luffy_moe_few: a whole mixture-of-experts layer for a step of a few tokens,
//   l_t = W_g x_t + b,  (e_tj, g_tj) = top-k of softmax(l_t),
//   h_tj = act(W1_e x_t),  y_t = sum_j g_tj W2_e h_tj,   e = e_tj.
// Every expert in use is a product of a few rows, so the layer is bound by
// reading the weights of those experts once; tokens, hidden rows and results
// are small beside them.
//
// Three launches: few_gate_kernel (a block a token: logits in float64, top-k,
// gates), few_product_kernel<.., false> (hidden rows) and <.., true> (second
// product, whose last block of each column tile adds the tokens' experts).
#include "act.h"
#include "luffy_common.h"

namespace luffy {
namespace {

constexpr int kFewTokens = LUFFY_FEW_MAX_TOKENS;
constexpr int kGateThreads = 1024;

enum FewWeights { kF32 = 0, kBf16 = 1, kMx4 = 2 };

// One block a token; wave w takes experts w, w + 16, ...  A logit is one
// float64 sum (products of two bf16 or float32 values are exact there), so a
// choice needs no second look at close calls.  Logits that are no number
// count below every other; a token without a single finite logit has gates of
// its own making (NaN, as softmax gives) but valid experts.
//
// With xs (4-bit weights) the block also stores its token's values in the
// order the 4-bit product takes them: of every 256 values (padded with zeros),
// value 32 c + 8 s + j at 64 s + 8 c + j, so that the eight lanes that hold a
// row's eight blocks read 128 contiguous bytes.
template <bool F32>
__global__ __launch_bounds__(kGateThreads) void few_gate_kernel(const void* __restrict__ x, int d,
                                                                const void* __restrict__ w_gate,
                                                                const float* __restrict__ b_gate, int E, int k,
                                                                int32_t* __restrict__ topk_idx,
                                                                float* __restrict__ topk_gate,
                                                                uint16_t* __restrict__ xs, int* __restrict__ done,
                                                                int n_done) {
  __shared__ double logit[kMaxExperts];
  const int t = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const size_t row = static_cast<size_t>(t) * d;
  for (int i = t * kGateThreads + tid; i < n_done; i += gridDim.x * kGateThreads) done[i] = 0;
  for (int e = w; e < E; e += kGateThreads / 64) {
    const size_t wrow = static_cast<size_t>(e) * d;
    double s = 0.0;
    if constexpr (F32) {
      for (int c = lane * 4; c < d; c += 256) {
        const float4 a = *reinterpret_cast<const float4*>(static_cast<const float*>(x) + row + c);
        const float4 b = *reinterpret_cast<const float4*>(static_cast<const float*>(w_gate) + wrow + c);
        s = fma(static_cast<double>(a.x), static_cast<double>(b.x), s);
        s = fma(static_cast<double>(a.y), static_cast<double>(b.y), s);
        s = fma(static_cast<double>(a.z), static_cast<double>(b.z), s);
        s = fma(static_cast<double>(a.w), static_cast<double>(b.w), s);
      }
    } else {
      for (int c = lane * 8; c < d; c += 512) {
        Pack16 a, b;
        a.u4 = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(x) + row + c);
        b.u4 = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(w_gate) + wrow + c);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          s = fma(static_cast<double>(bf16_to_f32(a.h[i])), static_cast<double>(bf16_to_f32(b.h[i])), s);
      }
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o, 64);
    if (lane == 0) logit[e] = s + (b_gate ? static_cast<double>(b_gate[e]) : 0.0);
  }
  if (xs) {
    const int pitch = (d + 255) / 256 * 256;
    uint16_t* dst = xs + static_cast<size_t>(t) * pitch;
    for (int i = tid * 8; i < pitch; i += kGateThreads * 8) {
      const int s = i >> 6 & 3, c = i >> 3 & 7, src = (i & ~255) + 32 * c + 8 * s;
      uint4 v = make_uint4(0, 0, 0, 0);
      if (src < d) v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(x) + row + src);
      *reinterpret_cast<uint4*>(dst + i) = v;
    }
  }
  __syncthreads();
  if (w != 0) return;
  const double mine = lane < E ? logit[lane] : 0.0;
  const bool num = lane < E && !isnan(mine);
  double v0 = 0.0, v1 = 0.0;
  int i0 = 0, i1 = 0;
  // largest first, ties to the lower index; taken marks experts already chosen
  uint64_t taken = 0;
  for (int j = 0; j < k; ++j) {
    const bool open = lane < E && !(taken >> lane & 1);
    double best = open && num ? mine : -HUGE_VAL;
    int at = open ? lane : kMaxExperts;
    bool bn = open && num;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double ob = __shfl_xor(best, o, 64);
      const int oa = __shfl_xor(at, o, 64);
      const bool on = __shfl_xor(static_cast<int>(bn), o, 64);
      const bool take = oa < kMaxExperts &&
                        (at == kMaxExperts || (on != bn ? on : (ob > best || (ob == best && oa < at))));
      if (take) { best = ob; at = oa; bn = on; }
    }
    taken |= 1ull << at;
    const double v = logit[at];
    if (j == 0) { i0 = at; v0 = v; } else { i1 = at; v1 = v; }
  }
  if (k == 1) {
    float den = lane < E ? expf(static_cast<float>(mine - v0)) : 0.f;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) den += __shfl_xor(den, o, 64);
    if (lane == 0) {
      topk_idx[t] = i0;
      topk_gate[t] = 1.0f / den;
    }
  } else if (lane == 0) {
    const float r = expf(static_cast<float>(v1 - v0));
    topk_idx[2 * t] = i0;
    topk_idx[2 * t + 1] = i1;
    topk_gate[2 * t] = 1.0f / (1.0f + r);
    topk_gate[2 * t + 1] = r / (1.0f + r);
  }
}

// Which slots (token t, choice j: t * k + j) expert number `rank` of the
// experts in use has; block-uniform.  Returns false when fewer are in use.
struct FewLists {
  int flag[kMaxExperts];
  int slot[kFewTokens];
  int count;
};

__device__ __forceinline__ bool few_expert(const int32_t* __restrict__ topk_idx, int slots, int rank, FewLists& l,
                                           int& e, int& n, int& used) {
  const int tid = threadIdx.x, lane = tid & 63;
  if (tid < kMaxExperts) l.flag[tid] = 0;
  __syncthreads();
  for (int i = tid; i < slots; i += blockDim.x) l.flag[topk_idx[i]] = 1;
  __syncthreads();
  const uint64_t m = __ballot(l.flag[lane] != 0);
  used = __popcll(m);
  if (rank >= used) return false;
  const uint64_t hit = __ballot((m >> lane & 1) && __popcll(m & lanemask_lt()) == rank);
  e = __builtin_amdgcn_readfirstlane(__builtin_ctzll(hit));
  if (tid < 64) {
    int base = 0;
    for (int s0 = 0; s0 < slots; s0 += 64) {
      const bool mine = s0 + lane < slots && topk_idx[s0 + lane] == e;
      const uint64_t b = __ballot(mine);
      const int at = base + __popcll(b & lanemask_lt());
      if (mine && at < kFewTokens) l.slot[at] = s0 + lane;   // a token has an expert at most once
      base += __popcll(b);
    }
    if (lane == 0) l.count = base;
  }
  __syncthreads();
  n = min(l.count, kFewTokens);
  return true;
}

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ bf16x8 mx4_to_bf16(uint32_t q, float scale) {
  typedef __bf16 bf16v2 __attribute__((ext_vector_type(2)));
  union { bf16v2 p[4]; bf16x8 v; } r;
  r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, scale, 0);
  r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, scale, 1);
  r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, scale, 2);
  r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, scale, 3);
  return r.v;
}

// The 8 x 8 products of one 128-byte piece of eight weight rows with eight
// tokens, on 16 x 16 MFMA.  Lane l holds 16 bytes of row l % 8, chunk l / 8 (so
// one load instruction reads eight whole 128-byte lines, the pattern that
// streams fastest: 6.9 TB/s of reads against 6.2 for 64-byte pieces).  Seen as
// an MFMA operand, rows 0-7 of a lane quarter g hold chunk 2g and rows 8-15
// the same weight rows' chunk 2g + 1, and the tokens come the same way, so
//   product of row r, token c  =  D[r][c] + D[r + 8][c + 8];
// the other two quadrants mix chunks and are not used.
template <int WT, bool HILO>
__device__ __forceinline__ void few_mma(u32x4 a, float scale, const u32x4* b, f32x4& acc) {
  if constexpr (WT == kF32) {
    const f32x4 av = __builtin_bit_cast(f32x4, a), bv = __builtin_bit_cast(f32x4, b[0]);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(av[i], bv[i], acc, 0, 0, 0);
  } else if constexpr (WT == kBf16) {
    const bf16x8 av = __builtin_bit_cast(bf16x8, a);
    acc = mfma16x16x32(av, __builtin_bit_cast(bf16x8, b[0]), acc);
    if constexpr (HILO) acc = mfma16x16x32(av, __builtin_bit_cast(bf16x8, b[1]), acc);
  } else {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const bf16x8 av = mx4_to_bf16(a[s], scale);
      acc = mfma16x16x32(av, __builtin_bit_cast(bf16x8, b[s]), acc);
      if constexpr (HILO) acc = mfma16x16x32(av, __builtin_bit_cast(bf16x8, b[4 + s]), acc);
    }
  }
}

struct FewArgs {
  const void* w;            // [E, N, K] weights (4-bit: two a byte)
  const uint8_t* scale;     // [E, ceil(K/256), N, 8] (4-bit weights)
  const void* in;           // rows of `pitch` bytes: tokens (first product), slots (second)
  size_t lo;                // second product: byte offset of the low halves of `in`
  int pitch;
  int N, K;
  int T, k;
  const int32_t* topk_idx;
  const float* topk_gate;
  void* h;                  // first product: hidden rows [slot], h_pitch bytes each
  size_t h_lo;
  int h_pitch;
  float* part;              // second product: [slot, N]
  int* done;                // a counter a column tile
  void* y;
};

// Position of hidden column c in a row of the second product's input.
template <int WT>
__device__ __forceinline__ int few_hidden_at(int c) {
  if constexpr (WT == kMx4) return (c & ~255) + 64 * (c >> 3 & 3) + 8 * (c >> 5 & 7) + (c & 7);
  else return c;
}

// One block: RT * 8 weight rows of one expert times that expert's tokens, K
// split over its W waves.  NB: groups of eight tokens a pass over the weights
// (an expert with more tokens passes over its rows again, from L2).
template <int WT, int RT, int W, int NB, bool SECOND>
__device__ __forceinline__ void few_tile(const FewArgs& a, int e, int n0, int first, int n, const int* slot,
                                         float* red, int act) {
  constexpr int U = RT >= 4 ? 2 : 4;                     // pieces of 128 bytes in flight a row
  constexpr bool HILO = SECOND && WT != kF32;
  constexpr int BP = (WT == kMx4 ? 4 : 1);               // 16-byte loads a lane, group and piece (and half)
  constexpr int BL = BP * (HILO ? 2 : 1);
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 7, c = lane >> 3;
  const int kbytes = WT == kF32 ? a.K * 4 : (WT == kBf16 ? a.K * 2 : a.K / 2);
  const int pieces = (kbytes + 127) / 128;
  const char* wp = static_cast<const char*>(a.w) + (static_cast<size_t>(e) * a.N + n0 + r) * kbytes + 16 * c;
  const uint8_t* sp = nullptr;
  if constexpr (WT == kMx4) sp = a.scale + (static_cast<size_t>(e) * pieces * a.N + n0 + r) * 8 + c;
  const char* bp[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int s = slot[min(first + 8 * b + r, n - 1)];
    bp[b] = static_cast<const char*>(a.in) + static_cast<size_t>(SECOND ? s : s / a.k) * a.pitch + 16 * c;
  }
  f32x4 acc[RT][NB];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int p0 = w * pieces / W, p1 = (w + 1) * pieces / W;
  for (int p = p0; p < p1; p += U) {
    u32x4 av[U][RT];
    float sv[U][RT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        av[u][i] = u32x4{0, 0, 0, 0};
        sv[u][i] = 0.f;
        // chunks past the row's end (K no multiple of 256) hold zeros
        if (p + u < p1 && (WT != kMx4 || (p + u) * 128 + 16 * c < kbytes)) {
          av[u][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(
              wp + static_cast<size_t>(8 * i) * kbytes + static_cast<size_t>(p + u) * 128));
          if constexpr (WT == kMx4) {
            const uint32_t s8 = sp[(static_cast<size_t>(p + u) * a.N + 8 * i) * 8];
            sv[u][i] = __uint_as_float(s8 << 23);   // only the exponent is read; 255 gives NaN
          }
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (p + u < p1) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          u32x4 bv[BL];
#pragma unroll
          for (int q = 0; q < BL; ++q) bv[q] = u32x4{0, 0, 0, 0};
          // (hidden rows have nothing past the last column)
          if (WT != kMx4 || (p + u) * 128 + 16 * c < kbytes) {
#pragma unroll
            for (int q = 0; q < BP; ++q) {
              const char* at = bp[b] + (static_cast<size_t>(p + u) * BP + q) * 128;
              bv[q] = *reinterpret_cast<const u32x4*>(at);
              if constexpr (HILO) bv[BP + q] = *reinterpret_cast<const u32x4*>(at + a.lo);
            }
          }
#pragma unroll
          for (int i = 0; i < RT; ++i) few_mma<WT, HILO>(av[u][i], sv[u][i], bv, acc[i][b]);
        }
      }
    }
  }
  // D[r][c] (lanes 0-7 and 16-23) + D[r + 8][c + 8] (40 lanes further), then
  // the waves' parts in wave order
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float other = __shfl(acc[i][b][v], (lane + 40) & 63, 64);
        if ((lane & 8) == 0 && lane < 32)
          red[((w * NB + b) * 8 + (lane & 7)) * (RT * 8) + 8 * i + 4 * (lane >> 4) + v] = acc[i][b][v] + other;
      }
  __syncthreads();
  for (int o = threadIdx.x; o < NB * 8 * RT * 8; o += W * 64) {
    const int col = o % (RT * 8), tok = o / (RT * 8);
    if (first + tok < n) {
      float z = 0.f;
#pragma unroll
      for (int q = 0; q < W; ++q) z += red[(q * NB * 8 + tok) * (RT * 8) + col];
      const int s = slot[first + tok];
      if constexpr (SECOND) {
        // read by whichever block adds this tile's experts, maybe on another XCD
        __hip_atomic_store(a.part + static_cast<size_t>(s) * a.N + n0 + col, z * a.topk_gate[s], __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
      } else {
        const float hv = act == LUFFY_ACT_GELU ? act_f32<LUFFY_ACT_GELU>(z) : act_f32<LUFFY_ACT_SILU>(z);
        char* dst = static_cast<char*>(a.h) + static_cast<size_t>(s) * a.h_pitch;
        const int at = few_hidden_at<WT>(n0 + col);
        if constexpr (WT == kF32) {
          reinterpret_cast<float*>(dst)[at] = hv;
        } else {
          // hidden rows stay float32 in effect: two bf16 halves whose sum is
          // within 2^-17 of the value, multiplied one after the other
          const uint32_t hi = pack_bf16x2(hv, 0.f) & 0xFFFFu;
          float rest = hv - __uint_as_float(hi << 16);
          if (!(fabsf(rest) < HUGE_VALF)) rest = 0.f;   // an infinite or NaN value is all in its high half
          reinterpret_cast<uint16_t*>(dst)[at] = static_cast<uint16_t>(hi);
          reinterpret_cast<uint16_t*>(dst + a.h_lo)[at] = static_cast<uint16_t>(pack_bf16x2(rest, 0.f) & 0xFFFFu);
        }
      }
    }
  }
  __syncthreads();
}

template <int WT, int RT, int W, bool SECOND>
__global__ __launch_bounds__(W * 64) void few_product_kernel(const FewArgs a, int act) {
  __shared__ FewLists lists;
  __shared__ float red[W * 4 * 8 * RT * 8];
  __shared__ int last;
  const int tiles = a.N / (RT * 8), tile = blockIdx.x % tiles;
  int e, n, used;
  if (!few_expert(a.topk_idx, a.T * a.k, blockIdx.x / tiles, lists, e, n, used)) return;
  const int n0 = tile * RT * 8;
  for (int first = 0; first < n; first += 32) {
    const int left = n - first;
    if (left <= 8) few_tile<WT, RT, W, 1, SECOND>(a, e, n0, first, n, lists.slot, red, act);
    else if (left <= 16) few_tile<WT, RT, W, 2, SECOND>(a, e, n0, first, n, lists.slot, red, act);
    else few_tile<WT, RT, W, 4, SECOND>(a, e, n0, first, n, lists.slot, red, act);
  }
  if constexpr (SECOND) {
    // every wave waits for its own partial results, then the block counts
    // itself done; the last of a tile's experts adds them in slot order
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0)
      last = __hip_atomic_fetch_add(a.done + tile, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == used - 1;
    __syncthreads();
    if (!last) return;
    for (int o = threadIdx.x; o < a.T * RT * 8; o += W * 64) {
      const int t = o / (RT * 8), col = n0 + o % (RT * 8);
      float v = 0.f;
      for (int j = 0; j < a.k; ++j)
        v += __hip_atomic_load(a.part + static_cast<size_t>(t * a.k + j) * a.N + col, __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT);
      if constexpr (WT == kF32) static_cast<float*>(a.y)[static_cast<size_t>(t) * a.N + col] = v;
      else static_cast<uint16_t*>(a.y)[static_cast<size_t>(t) * a.N + col] =
          static_cast<uint16_t>(pack_bf16x2(v, 0.f) & 0xFFFFu);
    }
  }
}

struct FewWs {
  uint16_t* xs;    // 4-bit weights: tokens in the product's order
  char* h;         // hidden rows, then (bf16, 4-bit) their low halves
  float* part;
  int* done;
};

// rows padded to whole 256 values, so one layout serves every weight type
FewWs carve_few(Carver& c, int T, int d, int k, int d_ff) {
  const size_t dp = align_up(d, 256), fp = align_up(d_ff, 256);
  FewWs w;
  w.xs = c.take<uint16_t>(static_cast<size_t>(T) * dp);
  w.h = c.take<char>(static_cast<size_t>(T) * k * fp * 4);
  w.part = c.take<float>(static_cast<size_t>(T) * k * d);
  w.done = c.take<int>(d / 8);
  return w;
}

template <int WT, int RT, bool SECOND>
void launch_few(const FewArgs& a, int experts, int act, hipStream_t s) {
  launch(SECOND ? "few_ffn2" : "few_ffn1", few_product_kernel<WT, RT, 4, SECOND>, experts * (a.N / (RT * 8)), 256, 0,
         s, a, act);
}

template <int WT>
void run_few(const void* x, int T, int d, const void* w_gate, const float* b_gate, int E, int k, const void* w1,
             const uint8_t* s1, const void* w2, const uint8_t* s2, int d_ff, int act, int32_t* topk_idx,
             float* topk_gate, void* y, const FewWs& ws, hipStream_t s) {
  launch("few_gate", few_gate_kernel<WT == kF32>, T, kGateThreads, 0, s, x, d, w_gate, b_gate, E, k, topk_idx,
         topk_gate, WT == kMx4 ? ws.xs : nullptr, ws.done, d / 8);
  const int experts = E < T * k ? E : T * k;
  const size_t fp = align_up(d_ff, 256);
  FewArgs a = {};
  a.T = T;
  a.k = k;
  a.topk_idx = topk_idx;
  a.topk_gate = topk_gate;
  a.w = w1;
  a.scale = s1;
  a.in = WT == kMx4 ? static_cast<const void*>(ws.xs) : x;
  a.pitch = WT == kF32 ? d * 4 : (WT == kBf16 ? d * 2 : static_cast<int>(align_up(d, 256)) * 2);
  a.N = d_ff;
  a.K = d;
  a.h = ws.h;
  a.h_pitch = static_cast<int>(WT == kF32 ? fp * 4 : fp * 2);
  a.h_lo = static_cast<size_t>(T) * k * fp * 2;
  launch_few<WT, 2, false>(a, experts, act, s);
  a.w = w2;
  a.scale = s2;
  a.in = ws.h;
  a.pitch = a.h_pitch;
  a.lo = a.h_lo;
  a.N = d;
  a.K = d_ff;
  a.part = ws.part;
  a.done = ws.done;
  a.y = y;
  launch_few<WT, 2, true>(a, experts, act, s);
}

bool few_misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

}  // namespace
}  // namespace luffy

using namespace luffy;

extern "C" size_t luffy_moe_few_workspace_size(int T, int d, int E, int k, int d_ff) {
  if (T <= 0 || T > kFewTokens || d <= 0 || E <= 0 || (k != 1 && k != 2) || d_ff <= 0) return 0;
  Carver c(nullptr);
  carve_few(c, T, d, k, d_ff);
  return c.size();
}

extern "C" int luffy_moe_few(const void* x, int T, int d, int dtype, const void* w_gate, const float* b_gate, int E,
                             int k, const void* w1, const void* w1_scale, const void* w2, const void* w2_scale,
                             int weight_type, int d_ff, int act, int32_t* topk_idx, float* topk_gate, void* y,
                             void* workspace, size_t workspace_bytes, void* stream) {
  if (!x || !w_gate || !w1 || !w2 || !topk_idx || !topk_gate || !y)
    return fail(LUFFY_E_INVALID, "luffy_moe_few: null pointer argument");
  if (T <= 0 || d <= 0 || E <= 0 || d_ff <= 0)
    return fail(LUFFY_E_INVALID, "luffy_moe_few: T=%d d=%d E=%d d_ff=%d", T, d, E, d_ff);
  if ((k != 1 && k != 2) || k > E) return fail(LUFFY_E_INVALID, "luffy_moe_few: k=%d must be 1 or 2 and at most E", k);
  if (dtype != LUFFY_F32 && dtype != LUFFY_BF16)
    return fail(LUFFY_E_INVALID, "luffy_moe_few: unknown dtype %d", dtype);
  if (weight_type != dtype && weight_type != LUFFY_MX4)
    return fail(LUFFY_E_INVALID, "luffy_moe_few: weight type %d with activations of type %d", weight_type, dtype);
  if (weight_type == LUFFY_MX4 && dtype != LUFFY_BF16)
    return fail(LUFFY_E_UNSUPPORTED, "luffy_moe_few: 4-bit weights take bf16 activations");
  if (weight_type == LUFFY_MX4 && (!w1_scale || !w2_scale))
    return fail(LUFFY_E_INVALID, "luffy_moe_few: 4-bit weights need their scales");
  if (act != LUFFY_ACT_GELU && act != LUFFY_ACT_SILU)
    return fail(LUFFY_E_INVALID, "luffy_moe_few: unknown activation %d", act);
  if (T > kFewTokens) return fail(LUFFY_E_UNSUPPORTED, "luffy_moe_few: T=%d > %d tokens", T, kFewTokens);
  if (E > kMaxExperts) return fail(LUFFY_E_UNSUPPORTED, "luffy_moe_few: E=%d > %d", E, kMaxExperts);
  if (d % 64 != 0 || d_ff % 64 != 0 || d > 32768 || d_ff > 32768)
    return fail(LUFFY_E_UNSUPPORTED, "luffy_moe_few: d=%d d_ff=%d must be multiples of 64 and at most 32768", d, d_ff);
  if (few_misaligned(x) || few_misaligned(w_gate) || few_misaligned(w1) || few_misaligned(w2))
    return fail(LUFFY_E_INVALID, "luffy_moe_few: x, w_gate, w1 and w2 must be 16-byte aligned");
  const size_t need = luffy_moe_few_workspace_size(T, d, E, k, d_ff);
  if (workspace_bytes < need || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return fail(LUFFY_E_WORKSPACE, "luffy_moe_few: workspace needs %zu bytes, 256-aligned", need);
  hipStream_t s = static_cast<hipStream_t>(stream);
  Carver c(workspace);
  const FewWs ws = carve_few(c, T, d, k, d_ff);
  const auto* s1 = static_cast<const uint8_t*>(w1_scale);
  const auto* s2 = static_cast<const uint8_t*>(w2_scale);
  if (weight_type == LUFFY_F32)
    run_few<kF32>(x, T, d, w_gate, b_gate, E, k, w1, s1, w2, s2, d_ff, act, topk_idx, topk_gate, y, ws, s);
  else if (weight_type == LUFFY_BF16)
    run_few<kBf16>(x, T, d, w_gate, b_gate, E, k, w1, s1, w2, s2, d_ff, act, topk_idx, topk_gate, y, ws, s);
  else
    run_few<kMx4>(x, T, d, w_gate, b_gate, E, k, w1, s1, w2, s2, d_ff, act, topk_idx, topk_gate, y, ws, s);
  return check_launch("luffy_moe_few");
}
