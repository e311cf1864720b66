// luffy_moe_few: a whole mixture-of-experts layer for a step of a few tokens,
//   l_t = W_g x_t + b,  (e_tj, g_tj) = top-k of softmax(l_t),
//   h_tj = act(W1_e x_t),  y_t = sum_j g_tj W2_e h_tj,   e = e_tj.
// Every expert in use is a product of a few rows, so the layer is bound by
// reading the weights of those experts once; tokens, hidden rows and results
// are small beside them.
//
// Three launches: few_gate_kernel (a block a token: logits in float64, top-k,
// gates), the hidden rows, and the second product, which also adds the tokens'
// experts; the products by few_product_kernel, or by few_direct_kernel for the
// fewest tokens.
#include <algorithm>

#include "act.h"
#include "luffy_common.h"
#include "mx4_core.h"

namespace luffy {
namespace {

constexpr int kFewTokens = LUFFY_FEW_MAX_TOKENS;
constexpr int kGateThreads = 1024;
constexpr int kFewWaves = 8, kFewThreads = 64 * kFewWaves;
constexpr int kDirectSlots = 8;   // few_direct_kernel's most
constexpr int kTiles = 2;         // few_product_kernel: tiles of eight rows that a wave has

enum FewWeights { kF32 = 0, kBf16 = 1, kMx4 = 2 };

// The tokens' side of the products ("columns") is kept in rows of 128-byte
// units: BL units for every 128-byte piece of a weight row.
//   float32           1 unit: the 32 values
//   bf16, tokens      1 unit: the 64 values
//   bf16, hidden      2 units: the 64 values' bf16 parts and what those leave
//                     (also bf16), together 16 bits of every float32 value
//   4-bit             2 units a term: 256 values as E4M3 with a scale byte per
//                     32, term t the E4M3 rounding of what the terms before
//                     leave, at 2^-4t of the scale.  Two terms hold a bf16 token
//                     exactly (but for values below 2^-13 of their block's
//                     largest, to 2^-21 of it), three hold a hidden value to
//                     2^-12 of itself or 2^-25 of its block's largest.  So the
//                     weights' codes go to the block-scaled MFMA as they are,
//                     without a conversion to bf16 for every value.
template <int WT, bool SECOND>
struct FewLayout {
  static constexpr int TERMS = SECOND ? 3 : 2;
  static constexpr int BL = WT == kMx4 ? 2 * TERMS : (WT == kBf16 && SECOND ? 2 : 1);
  static constexpr int PIECE = WT == kF32 ? 32 : (WT == kBf16 ? 64 : 256);   // values of a piece
};
template <int WT, bool SECOND>
__host__ __device__ constexpr int few_pitch(int K) {
  return (K + FewLayout<WT, SECOND>::PIECE - 1) / FewLayout<WT, SECOND>::PIECE * FewLayout<WT, SECOND>::BL * 128;
}
__host__ __device__ constexpr int few_scale_pitch(int K) { return (K + 255) / 256 * 8; }

// Stores eight consecutive values (unit `u` of eight of a row; the four units
// of a block of 32 sit in four neighbouring lanes) as TERMS E4M3 terms.  The
// block-scaled MFMA 16x16x128 takes 8-bit values k = 64 h + 16 g + b from byte
// 16 h + b of lane quarter g, and the scale of values 32 g.. from quarter g (4-
// bit values: 32 g.. in quarter g).  The weight blocks a lane holds put block
// c of a piece at quarter c / 2 of the half c % 2 of a wave's rows, so value i
// of block c goes to half h = c / 4, eighth 4 (c / 2 % 2) + 2 (i / 16) + c % 2.
template <int TERMS>
__device__ __forceinline__ void store_e4m3(float (&v)[8], int u, uint8_t* __restrict__ row, uint8_t* __restrict__ scale) {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  typedef float f32v2 __attribute__((ext_vector_type(2)));
  uint32_t most = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(v[j]) & 0x7fffffffu);
  most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 1, 64)));
  most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 2, 64)));
  // largest value in [128, 256) of the first scale; 4 (TERMS - 1) is left below it
  const uint32_t ex = most >> 23, s0 = ex == 255u ? 255u : max(static_cast<int>(ex) - 7, 8);
  const int c = u >> 2 & 7, j = u & 3, piece = u >> 5;
  const int at = 128 * (c >> 2) + 16 * (4 * (c >> 1 & 1) + 2 * (j >> 1) + (c & 1)) + 8 * (j & 1);
#pragma unroll
  for (int t = 0; t < TERMS; ++t) {
    const float sc = __uint_as_float((s0 - 4 * t) << 23);
    s16x2 q[2] = {{0, 0}, {0, 0}};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      q[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q[i], v[4 * i], v[4 * i + 1], sc, false);
      q[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q[i], v[4 * i + 2], v[4 * i + 3], sc, true);
    }
    const int w0 = __builtin_bit_cast(int, q[0]), w1 = __builtin_bit_cast(int, q[1]);
    if (t + 1 < TERMS) {
      const f32v2 b0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w0, sc, false);
      const f32v2 b1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w0, sc, true);
      const f32v2 b2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w1, sc, false);
      const f32v2 b3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w1, sc, true);
      v[0] -= b0.x; v[1] -= b0.y; v[2] -= b1.x; v[3] -= b1.y;
      v[4] -= b2.x; v[5] -= b2.y; v[6] -= b3.x; v[7] -= b3.y;
    }
    const uint2 o = ex == 255u ? make_uint2(0, 0) : make_uint2(w0, w1);
    *reinterpret_cast<uint2*>(row + (static_cast<size_t>(piece) * 2 * TERMS + 2 * t) * 128 + at) = o;
  }
  if (j == 0) scale[piece * 8 + c] = static_cast<uint8_t>(s0);
}

struct FewTerms {   // 4-bit weights: the tokens' and hidden rows' terms and scales
  uint8_t *x8, *x8_scale, *h8, *h8_scale;
  int d_ff;
};

template <int CTRL>
__device__ __forceinline__ double add_dpp(double v) {
  const int2 a = __builtin_bit_cast(int2, v);
  const int2 b = make_int2(__builtin_amdgcn_update_dpp(0, a.x, CTRL, 0xf, 0xf, true),
                           __builtin_amdgcn_update_dpp(0, a.y, CTRL, 0xf, 0xf, true));
  return v + __builtin_bit_cast(double, b);
}
// Sum over a wave, in every lane, without going through LDS: neighbours, pairs,
// fours and eights by row permutations, rows of 16 and halves by swaps.
__device__ __forceinline__ double sum64(double v) {
  v = add_dpp<0xB1>(v);    // lane ^ 1
  v = add_dpp<0x4E>(v);    // lane ^ 2
  v = add_dpp<0x141>(v);   // mirrored in 8
  v = add_dpp<0x140>(v);   // mirrored in 16
  uint2 a = __builtin_bit_cast(uint2, v);
  auto x = __builtin_amdgcn_permlane16_swap(a.x, a.x, false, false), y = __builtin_amdgcn_permlane16_swap(a.y, a.y, false, false);
  v = __builtin_bit_cast(double, make_uint2(x[0], y[0])) + __builtin_bit_cast(double, make_uint2(x[1], y[1]));
  a = __builtin_bit_cast(uint2, v);
  x = __builtin_amdgcn_permlane32_swap(a.x, a.x, false, false);
  y = __builtin_amdgcn_permlane32_swap(a.y, a.y, false, false);
  return __builtin_bit_cast(double, make_uint2(x[0], y[0])) + __builtin_bit_cast(double, make_uint2(x[1], y[1]));
}

// One block a token; wave w takes experts w, w + 16, ...  3.2 us for 7 tokens of
// 256 values on 4 experts, 6.3 for 64 of 4096 on 8: a launch and two trips to
// memory.  A logit is one
// float64 sum (products of two bf16 or float32 values are exact there), so a
// choice needs no second look at close calls.  Logits that are no number
// count below every other; a token without a single finite logit has gates of
// its own making (NaN, as softmax gives) but valid experts.
//
// With x8 (4-bit weights) the block also stores its token's values as E4M3
// terms (store_e4m3), zeros past the last one, and clears the last piece of its
// hidden rows h8, which the first product may fill only in part.
template <bool F32>
__global__ __launch_bounds__(kGateThreads) void few_gate_kernel(const void* __restrict__ x, int d,
                                                                const void* __restrict__ w_gate,
                                                                const float* __restrict__ b_gate, int E, int k,
                                                                int32_t* __restrict__ topk_idx,
                                                                float* __restrict__ topk_gate,
                                                                const FewTerms f, int* __restrict__ done,
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
    s = sum64(s);
    if (lane == 0) logit[e] = s + (b_gate ? static_cast<double>(b_gate[e]) : 0.0);
  }
  if (f.x8) {
    uint8_t* dst = f.x8 + static_cast<size_t>(t) * few_pitch<kMx4, false>(d);
    uint8_t* scale = f.x8_scale + static_cast<size_t>(t) * few_scale_pitch(d);
    const int units = (d + 255) / 256 * 32;   // a multiple of 32: a block's four lanes stay together
    for (int u = tid; u < units; u += kGateThreads) {
      Pack16 a;
      a.u4 = make_uint4(0, 0, 0, 0);
      if (u * 8 < d) a.u4 = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(x) + row + u * 8);
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = bf16_to_f32(a.h[i]);
      store_e4m3<2>(v, u, dst, scale);
    }
    if (f.d_ff & 255) {
      constexpr int words = FewLayout<kMx4, true>::BL * 32;
      for (int i = tid; i < k * words; i += kGateThreads) {
        const int slot = t * k + i / words;
        uint8_t* end = f.h8 + static_cast<size_t>(slot + 1) * few_pitch<kMx4, true>(f.d_ff) - 4 * words;
        reinterpret_cast<uint32_t*>(end)[i % words] = 0;
      }
      if (tid < 2 * k)
        reinterpret_cast<uint32_t*>(f.h8_scale + static_cast<size_t>(t * k + tid / 2 + 1) * few_scale_pitch(f.d_ff) -
                                    8)[tid & 1] = 0;
    }
  }
  __syncthreads();
  if (w != 0) return;
  const double mine = lane < E ? logit[lane] : 0.0;
  // An expert's rank: how many come before it (larger first, ties to the lower
  // index, no number last).  Its logit becomes an integer of the same order, 0
  // for no number, and every lane compares its own with each in turn.
  const uint64_t bits = __builtin_bit_cast(uint64_t, mine + 0.0);   // (-0 + 0 = +0: the two are a tie)
  const uint64_t sign = 1ull << 63;
  const uint64_t key = isnan(mine) ? 0 : (bits & sign ? ~bits : bits | sign);
  int rank = 0;
#pragma unroll 4
  for (int e = 0; e < E; ++e) {
    const uint64_t o = static_cast<uint64_t>(__builtin_amdgcn_readlane(static_cast<int>(key >> 32), e)) << 32 |
                       static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(key), e));
    rank += o >= key + (e >= lane ? 1 : 0) ? 1 : 0;
  }
  const int i0 = __ffsll(__ballot(lane < E && rank == 0)) - 1;
  const int i1 = k > 1 ? __ffsll(__ballot(lane < E && rank == 1)) - 1 : i0;
  const double v0 = logit[i0], v1 = logit[i1];
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

__device__ __forceinline__ void lds_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// The experts in use and their slots (token t, choice j: slot t * k + j).
struct FewLists {
  int expert[kMaxExperts], first[kMaxExperts + 1];   // by rank among the experts in use
  int slot[2 * kFewTokens];
  int used;
  int at[kMaxExperts];
};

// One wave.  The order of an expert's slots is that of the LDS atomics; it
// decides which column of the products a slot has and nothing else.
__device__ __forceinline__ void few_lists(const int32_t* __restrict__ topk_idx, int slots, FewLists& l) {
  const int lane = threadIdx.x & 63;
  const int e0 = lane < slots ? topk_idx[lane] : -1;
  const int e1 = 64 + lane < slots ? topk_idx[64 + lane] : -1;
  l.at[lane] = 0;
  lds_order();
  const int p0 = e0 >= 0 ? atomicAdd(&l.at[e0], 1) : 0;
  const int p1 = e1 >= 0 ? atomicAdd(&l.at[e1], 1) : 0;
  lds_order();
  const int n = l.at[lane];
  int incl = n;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(incl, o, 64);
    if (lane >= o) incl += v;
  }
  const uint64_t m = __ballot(n > 0);
  const int rank = __popcll(m & lanemask_lt());
  if (n > 0) {
    l.expert[rank] = lane;
    l.first[rank] = incl - n;
  }
  l.at[lane] = incl - n;
  if (lane == 63) {
    l.used = __popcll(m);
    l.first[__popcll(m)] = incl;
  }
  lds_order();
  if (e0 >= 0) l.slot[l.at[e0] + p0] = lane;
  if (e1 >= 0) l.slot[l.at[e1] + p1] = 64 + lane;
}

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// The 8 x 8 products of one 128-byte piece of eight weight rows with eight
// columns, on 16 x 16 MFMA.  Lane l holds 16 bytes of row l % 8, chunk l / 8 (so
// one load instruction reads eight whole 128-byte lines, the pattern that
// streams fastest: 6.9 TB/s of reads against 6.2 for 64-byte pieces).  Seen as
// an MFMA operand, rows 0-7 of a lane quarter g hold chunk 2g and rows 8-15
// the same weight rows' chunk 2g + 1, and the columns come the same way, so
//   product of row r, column c  =  D[r][c] + D[r + 8][c + 8];
// the other two quadrants mix chunks and are not used.
template <int WT, int BL>
__device__ __forceinline__ void few_mma(u32x4 a, int sa, const u32x4 (&b)[BL], int sb, f32x4& acc) {
  if constexpr (WT == kF32) {
    const f32x4 av = __builtin_bit_cast(f32x4, a), bv = __builtin_bit_cast(f32x4, b[0]);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(av[i], bv[i], acc, 0, 0, 0);
  } else if constexpr (WT == kBf16) {
#pragma unroll
    for (int i = 0; i < BL; ++i)
      acc = mfma16x16x32(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b[i]), acc);
  } else {
    const i32x4 q = __builtin_bit_cast(i32x4, a);
    const i32x8 av = __builtin_shufflevector(q, q, 0, 1, 2, 3, -1, -1, -1, -1);
#pragma unroll
    for (int t = 0; t < BL / 2; ++t) {
      const i32x4 lo = __builtin_bit_cast(i32x4, b[2 * t]), hi = __builtin_bit_cast(i32x4, b[2 * t + 1]);
      const i32x8 bv = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, bv, acc, 4, 0, 0, sa, 0, sb - 4 * t);
    }
  }
}

struct FewArgs {
  const uint8_t* w;         // [E, N, K] weights
  const uint8_t* w_scale;   // [E, ceil(K/256), N, 8] (4-bit weights)
  const uint8_t* in;        // columns: tokens (first product) or slots (second), FewLayout rows
  const uint8_t* in_scale;
  int N, K, T, k, split;    // split: waves that share a row's K (1, 2, 4 or 8)
  int groups;               // row groups of N: ceil(N / rows of an item)
  float per_group, per_block;   // 1 / groups, 1 / blocks
  const int32_t* topk_idx;
  const float* topk_gate;
  uint8_t *h, *h_scale;     // first product: hidden rows by slot
  float* part;              // second product: [slot, N]
  int* done;                // a counter a row group
  void* y;
};

// BYTES (4 or 16) a lane from offset off + soff to dst + BYTES * lane,
// asynchronously.
template <int BYTES>
__device__ __forceinline__ void lds_dma(__amdgpu_buffer_rsrc_t r, uint32_t off, int soff,
                                        __attribute__((address_space(3))) uint8_t* dst) {
  using lds_ptr = __attribute__((address_space(3))) void*;
  if constexpr (BYTES == 16) __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr)dst, 16, off, soff, 0, 0);
  else __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr)dst, 4, off, soff, 0, 0);
}

// Barrier for data in LDS: waits for this wave's LDS accesses only, so that
// loads from memory stay in flight across it.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  raw_barrier();
}

// LDS of a block.  Columns come in chunks of K, double-buffered; NBMAX: groups
// of eight columns that an item may have (an expert has at most T).  With one
// group the registers allow two blocks a CU, with more one.
template <int NBMAX>
struct FewLds {
  static constexpr int HALF = (NBMAX == 1 ? 24 : 48) * 1024;      // one chunk's columns
  static constexpr int SCALES = NBMAX == 1 ? 1024 : 2048;         // and their scale bytes (8 a piece and column)
  static constexpr int RED = NBMAX * 8 * kFewWaves * kTiles * 8 * 4;  // the waves' sums
  // float32 and bf16: the scales' place holds zeros for a piece of every column
  static constexpr int ZEROS_AT = 2 * HALF, ZEROS = NBMAX * 8 * 128 * 2;
  __attribute__((aligned(16))) uint8_t cols[2 * HALF];
  __attribute__((aligned(16))) uint8_t scales[2 * SCALES];
  __attribute__((aligned(16))) uint8_t wscale[kFewWaves][2][1024];   // 4-bit weights: each wave's scales
  __attribute__((aligned(16))) float red[RED / 4];
  FewLists l;
  int ready;                       // row groups that this block adds up at its end
  int group[kFewThreads];
};

// Columns that n columns are kept as, log2: 1, 2, 4 or 8 in the one group, else
// whole groups (2, 4 or 8 of them).
__host__ __device__ constexpr int few_cols_log2(int n) {
  return n <= 1 ? 0 : (n <= 2 ? 1 : (n <= 4 ? 2 : (n <= 8 ? 3 : (n <= 16 ? 4 : (n <= 32 ? 5 : 6)))));
}
// A half's bytes for each part of K (whole DMA instructions), and the pieces of
// a part in a chunk.
template <int NBMAX>
__host__ __device__ constexpr int few_part_bytes(int split_log2) {
  return (FewLds<NBMAX>::HALF >> split_log2) & ~1023;
}
template <int WT, bool SECOND, int NBMAX>
__host__ __device__ constexpr int few_chunk(int split_log2, int cols_log2) {
  const int fit = few_part_bytes<NBMAX>(split_log2) / (128 * FewLayout<WT, SECOND>::BL) >> cols_log2;
  const int scales = FewLds<NBMAX>::SCALES / 8 >> (split_log2 + cols_log2);
  return WT == kMx4 && scales < fit ? scales : fit;
}
// With K in one part every number of columns fits (the loops over chunks would
// not advance otherwise).
template <int NBMAX, int COLS_LOG2>
constexpr bool few_fits() {
  return few_chunk<kF32, true, NBMAX>(0, COLS_LOG2) >= 1 && few_chunk<kBf16, true, NBMAX>(0, COLS_LOG2) >= 1 &&
         few_chunk<kMx4, false, NBMAX>(0, COLS_LOG2) >= 1 && few_chunk<kMx4, true, NBMAX>(0, COLS_LOG2) >= 1;
}
using FewLdsOne = FewLds<1>;
using FewLdsMore = FewLds<8>;
static_assert(offsetof(FewLdsOne, scales) == FewLdsOne::ZEROS_AT && offsetof(FewLdsMore, scales) == FewLdsMore::ZEROS_AT &&
                  FewLdsOne::ZEROS_AT + FewLdsOne::ZEROS <= offsetof(FewLdsOne, red) &&
                  FewLdsMore::ZEROS_AT + FewLdsMore::ZEROS <= offsetof(FewLdsMore, red),
              "zeros in the scales' place");
static_assert(few_fits<1, 3>() && few_fits<8, 6>(), "a piece of every column in LDS");
static_assert(sizeof(FewLds<8>) <= 160 * 1024 && 2 * sizeof(FewLds<1>) <= 160 * 1024, "LDS");

// A block's waves are arranged as `split` parts of K by 8 / split row groups of
// 16 rows (kTiles tiles); a work item is the 128 / split rows of one expert that
// the block takes at a time, times all of that expert's columns.
struct FewItem {
  const uint8_t *w, *s;          // the expert's weights and scales
  uint32_t row;                  // this wave's first row
  int rank, group, first, n;
  int p0, p1;                    // pieces of K of this wave (none where its rows do not exist)
  int c1;                        // and the end of those in the first chunk
};

template <int WT>
__host__ __device__ __forceinline__ int few_kbytes(int K) { return WT == kF32 ? K * 4 : (WT == kBf16 ? K * 2 : K / 2); }

constexpr uint32_t kFewRange = 0xFFFF0000u;   // an expert's matrix is smaller (checked on the host)

__device__ __forceinline__ __amdgpu_buffer_rsrc_t few_rsrc(const uint8_t* base) {
  const uint64_t v = reinterpret_cast<uint64_t>(base);
  const uint64_t lo = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v)));
  const uint64_t hi = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v >> 32)));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((hi << 32) | lo), static_cast<short>(0),
                                           static_cast<int>(kFewRange), 0x00020000);
}

template <int WT, int NBMAX, bool SECOND>
__device__ __forceinline__ FewItem few_item(const FewArgs& a, const FewLists& l, int item) {
  FewItem t;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // item / groups: the product is off by less than one (items < 2^23)
  int rank = static_cast<int>(static_cast<float>(item) * a.per_group);
  if (rank * a.groups > item) --rank;
  if ((rank + 1) * a.groups <= item) ++rank;
  t.rank = __builtin_amdgcn_readfirstlane(rank);
  t.group = item - t.rank * a.groups;
  const int e = __builtin_amdgcn_readfirstlane(l.expert[t.rank]);
  t.first = __builtin_amdgcn_readfirstlane(l.first[t.rank]);
  t.n = __builtin_amdgcn_readfirstlane(l.first[t.rank + 1]) - t.first;
  const int kbytes = few_kbytes<WT>(a.K), pieces = (kbytes + 127) / 128, split_log2 = __builtin_ctz(a.split);
  const int part = w & (a.split - 1);
  t.row = (t.group * (kFewWaves >> split_log2) + (w >> split_log2)) * (8 * kTiles);
  const bool rows = static_cast<int>(t.row) < a.N;
  t.p0 = rows ? (part * pieces) >> split_log2 : 0;
  t.p1 = rows ? ((part + 1) * pieces) >> split_log2 : 0;
  t.c1 = min(t.p1, t.p0 + few_chunk<WT, SECOND, NBMAX>(split_log2, few_cols_log2(t.n)));
  t.w = a.w + static_cast<size_t>(e) * a.N * kbytes;
  t.s = WT == kMx4 ? a.w_scale + static_cast<size_t>(e) * pieces * a.N * 8 : nullptr;
  return t;
}

// U pieces of the wave's kTiles row tiles, from piece p on.  The loads are issued
// whatever p is, and those at or past p1 fetch nothing (their offset is out of
// the buffer's range; 4-bit: nor do chunks past the row's end) and give zeros:
// a load behind a branch would leave the number of loads in flight open, and
// every use of an earlier one would wait for all.
template <int WT, int U>
__device__ __forceinline__ void few_load(const FewArgs& a, const uint8_t* w, uint32_t row, int p, int p1,
                                         u32x4 (&av)[U][kTiles]) {
  constexpr int kStream = 2;   // non-temporal: read once
  const int kbytes = few_kbytes<WT>(a.K), lane = threadIdx.x & 63, r = lane & 7, c = lane >> 3;
  const uint32_t off = static_cast<uint32_t>(r) * kbytes + 16 * c;
  const __amdgpu_buffer_rsrc_t wr = few_rsrc(w);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t in = static_cast<uint32_t>((p + u - p1) >> 31);   // all ones where the piece exists
    uint32_t o = off | (~in & kFewRange);
    if constexpr (WT == kMx4) o = (p + u) * 128 + 16 * c < kbytes ? o : kFewRange;
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
      av[u][i] = __builtin_amdgcn_raw_buffer_load_b128(wr, o, ((row + 8 * i) * kbytes + (p + u) * 128) & in, kStream);
  }
}

// The scale bytes of the wave's 16 rows in eight pieces from piece p on, 128
// bytes a piece, into the wave's own LDS: one instruction in place of sixteen
// byte loads beside the weights' sixteen (pieces at or past p1: not fetched).
__device__ __forceinline__ void few_load_scales(const FewArgs& a, const uint8_t* s, uint32_t row, int p, int p1,
                                                __attribute__((address_space(3))) uint8_t* dst) {
  static_assert(kTiles == 2, "16 rows of 8 bytes, a lane quarter of 8 lanes each 16 bytes");
  const int lane = threadIdx.x & 63, u = lane >> 3;
  const uint32_t off = (static_cast<uint32_t>(u) * a.N + 2 * (lane & 7)) * 8;
  lds_dma<16>(few_rsrc(s), p + u < p1 ? off : kFewRange, p < p1 ? (p * a.N + row) * 8 : 0, dst);
  load_order();
}

// Values a thread finishes at a time: 4-bit weights' hidden rows are rounded
// eight at a time, everything else goes out in pairs (more threads at work).
template <int WT, bool SECOND>
constexpr int kFewValues = WT == kMx4 && !SECOND ? 8 : 2;

// Hidden values n, n + 1, ... of slot s from their sums z.
template <int WT>
__device__ __forceinline__ void few_store_hidden(const FewArgs& a, int act, int s, int n, bool valid,
                                                 float (&z)[kFewValues<WT, false>]) {
#pragma unroll
  for (int i = 0; i < kFewValues<WT, false>; ++i)
    z[i] = act == LUFFY_ACT_GELU ? act_f32_relative<LUFFY_ACT_GELU>(z[i]) : act_f32_relative<LUFFY_ACT_SILU>(z[i]);
  uint8_t* dst = a.h + static_cast<size_t>(s) * few_pitch<WT, true>(a.N);
  if constexpr (WT == kMx4) {
    // (a block's four lanes agree on valid: a block of waves has a multiple of
    // 32 rows and N is one of 64)
    if (valid) store_e4m3<3>(z, n / 8, dst, a.h_scale + static_cast<size_t>(s) * few_scale_pitch(a.N));
  } else if (valid) {
    if constexpr (WT == kF32) {
      *reinterpret_cast<float2*>(dst + n * 4) = make_float2(z[0], z[1]);
    } else {
      const uint32_t hi = pack_bf16x2(z[0], z[1]);
      float r0 = z[0] - __uint_as_float(hi << 16), r1 = z[1] - __uint_as_float(hi & 0xFFFF0000u);
      // an infinite or NaN value is all in its first part
      if (!(fabsf(r0) < HUGE_VALF)) r0 = 0.f;
      if (!(fabsf(r1) < HUGE_VALF)) r1 = 0.f;
      uint8_t* f = dst + (n >> 6) * 256 + (n & 63) * 2;
      *reinterpret_cast<uint32_t*>(f) = hi;
      *reinterpret_cast<uint32_t*>(f + 128) = pack_bf16x2(r0, r1);
    }
  }
}

// What the column buffers hold, and where the next chunk goes (block-uniform).
struct FewStage {
  int half;        // of the current chunk
  int whole;       // rank whose columns the half holds over all of K, -1: none
  bool behind;     // a step of weight loads follows the chunk's loads (this wave)
  int slot;        // of the current scales (this wave)
};

// Columns of the chunk of item t that starts at piece c0 of every part, straight
// into LDS (asynchronous loads, all in flight together): for every 128-byte
// unit of a part's pieces one line a column, a line's eighths permuted so that
// the products' reads (eight columns, one eighth) fall on distinct banks.  A
// DMA instruction fills eight lines.  Lines past the part's end are not
// fetched; nothing reads them.  The scale bytes of a column's chunk are one run.
template <int WT, int NB, int NBMAX, bool SECOND>
__device__ __forceinline__ void few_stage(const FewArgs& a, FewLds<NBMAX>& m, const FewItem& t, int c0, int half) {
  using S = FewLds<NBMAX>;
  using lds_ptr = __attribute__((address_space(3))) uint8_t*;
  constexpr int BL = FewLayout<WT, SECOND>::BL;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int pieces = (few_kbytes<WT>(a.K) + 127) / 128, pitch = few_pitch<WT, SECOND>(a.K);
  const int split_log2 = __builtin_ctz(a.split), cols_log2 = few_cols_log2(NB > 1 ? 8 * NB : t.n);
  const int chunk = few_chunk<WT, SECOND, NBMAX>(split_log2, cols_log2);
  const __amdgpu_buffer_rsrc_t in = few_rsrc(a.in);   // (a step's columns are far below 4 GiB)
  // this wave's part of K, one of the 8 / split waves that have it
  const int kp = w & (a.split - 1), first = ((kp * pieces) >> split_log2) + c0;
  const int len = min(chunk, (((kp + 1) * pieces) >> split_log2) - first), lines = len * BL << cols_log2;
  const lds_ptr cols = (lds_ptr)m.cols + half * S::HALF + kp * few_part_bytes<NBMAX>(split_log2);
  const int line = lane >> 3;
  uint32_t off[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int col = 8 * b + (line & ((1 << cols_log2) - 1));
    const int s = m.l.slot[t.first + min(col, t.n - 1)];
    off[b] = static_cast<uint32_t>(SECOND || a.k == 1 ? s : s >> 1) * pitch + 16 * ((lane & 7) ^ (col & 7));
    if (NB == 1) off[b] += (line >> cols_log2) * 128;
  }
#pragma unroll 1
  for (int l0 = (w >> split_log2) * (8 * NB); l0 < lines; l0 += (kFewWaves >> split_log2) * (8 * NB)) {
    const int soff = (first * BL + (l0 >> cols_log2)) * 128;
#pragma unroll
    for (int b = 0; b < NB; ++b)
      lds_dma<16>(in, NB > 1 || l0 + line < lines ? off[b] : kFewRange, soff, cols + (l0 + 8 * b) * 128);
  }
  if constexpr (WT == kMx4) {
    const __amdgpu_buffer_rsrc_t ins = few_rsrc(a.in_scale);
    const lds_ptr scales = (lds_ptr)m.scales + half * S::SCALES;
#pragma unroll 1
    for (int col = w >> split_log2; col < 1 << cols_log2; col += kFewWaves >> split_log2) {
      const int s = __builtin_amdgcn_readfirstlane(m.l.slot[t.first + min(col, t.n - 1)]);
      const uint32_t row = static_cast<uint32_t>(SECOND || a.k == 1 ? s : s >> 1) * few_scale_pitch(a.K) + first * 8;
      for (int d = 0; d < 2 * len; d += 64)
        if (d + lane < 2 * len)
          lds_dma<4>(ins, 4 * lane, row + 4 * d, scales + ((kp << cols_log2) + col) * chunk * 8 + 4 * d);
    }
  }
  load_order();
}

// Stages the first chunk of an item.
template <int WT, int NBMAX, bool SECOND>
__device__ __forceinline__ void few_stage_first(const FewArgs& a, FewLds<NBMAX>& m, const FewItem& t,
                                                int half) {
  if (NBMAX == 1 || t.n <= 8) few_stage<WT, 1, NBMAX, SECOND>(a, m, t, 0, half);
  else if (t.n <= 16) few_stage<WT, (NBMAX > 1 ? 2 : 1), NBMAX, SECOND>(a, m, t, 0, half);
  else if (t.n <= 32) few_stage<WT, (NBMAX > 1 ? 4 : 1), NBMAX, SECOND>(a, m, t, 0, half);
  else few_stage<WT, (NBMAX > 1 ? 8 : 1), NBMAX, SECOND>(a, m, t, 0, half);
}

// One work item with NB groups of eight columns.  av holds the item's first
// pieces on entry and the next item's (`next`, if any) on return, and its first
// columns are on their way to LDS, so that the weight stream does not stop
// while an item's sums are added and stored.
template <int WT, int NB, int NBMAX, bool SECOND>
__device__ __forceinline__ void few_run(const FewArgs& a, FewLds<NBMAX>& m, const FewItem& t,
                                        const FewItem& next, bool more, int act, FewStage& st,
                                        u32x4 (&av)[8 / kTiles][kTiles]) {
  using L = FewLayout<WT, SECOND>;
  using S = FewLds<NBMAX>;
  constexpr int U = 8 / kTiles, BL = L::BL;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int part = w & (a.split - 1), pieces = (few_kbytes<WT>(a.K) + 127) / 128;
  const int split_log2 = __builtin_ctz(a.split), cols_log2 = few_cols_log2(NB > 1 ? 8 * NB : t.n);
  const int chunk = few_chunk<WT, SECOND, NBMAX>(split_log2, cols_log2);
  const int span = (pieces + a.split - 1) >> __builtin_ctz(a.split);   // the longest part
  f32x4 acc[kTiles][NB];
#pragma unroll
  for (int i = 0; i < kTiles; ++i)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  using lds_ptr = __attribute__((address_space(3))) uint8_t*;
  const int lr = lane & 7, lc = lane >> 3, lane_scale = 8 * lr + lc;
#pragma unroll 1
  for (int c0 = 0; c0 < span; c0 += chunk) {
    if (c0 > 0 || st.whole != t.rank) {
      // this wave's columns have landed (all but its newest loads, a step of
      // weights); then every wave's, and every wave is done with the other half
      load_order();
      if (st.behind) wait_vmcnt<U * kTiles>();
      else wait_vmcnt<0>();
      lds_barrier();
      st.whole = span <= chunk ? t.rank : -1;
    }
    st.behind = false;
    if (c0 + chunk < span) {
      few_stage<WT, NB, NBMAX, SECOND>(a, m, t, c0 + chunk, st.half ^ 1);
    } else if (more && st.whole != next.rank) {
      few_stage_first<WT, NBMAX, SECOND>(a, m, next, st.half ^ 1);
    }
    // Steps of U pieces in pairs, the registers of one loaded while the other's
    // are multiplied; an odd number is filled up with a step that loads nothing.
    const int len = t.p1 - t.p0, end = min(len, c0 + chunk);
    const bool on = c0 + chunk < len;   // this wave has pieces in the next chunk
    // this lane's column in each group, and where its lines start
    const int lcol = lr & ((1 << cols_log2) - 1);
    const uint8_t* cols = reinterpret_cast<const uint8_t*>(&m) + lcol * 128 + 16 * (lc ^ (lcol & 7));
    const int cols_at = st.half * S::HALF + part * few_part_bytes<NBMAX>(split_log2);
    const uint8_t* scales = m.scales + st.half * S::SCALES + ((part << cols_log2) + lcol) * chunk * 8 + lc;
    // Pieces past the end are zeros, multiplied with zero columns (an infinity must
    // not meet a zero; 4-bit weights: with the last piece's columns under a zero
    // scale, where a block without numbers has made the result NaN already):
    // without branches the compiler knows how many loads are in flight.
    auto multiply = [&](const u32x4(&av)[U][kTiles], int p, const uint8_t* ws) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = min(p + u, end - 1) - c0;
        const int line = WT == kMx4 || p + u < end ? cols_at + ((at * BL) << cols_log2) * 128 : S::ZEROS_AT;
        int sa[kTiles];
#pragma unroll
        for (int i = 0; i < kTiles; ++i) sa[i] = WT == kMx4 ? ws[128 * u + 64 * i] & ((p + u - end) >> 31) : 0;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          u32x4 bv[BL];
          int sb = 0;
#pragma unroll
          for (int j = 0; j < BL; ++j)
            bv[j] = *reinterpret_cast<const u32x4*>(cols + line + ((j << cols_log2) + 8 * b) * 128);
          if constexpr (WT == kMx4) sb = scales[8 * b * chunk * 8 + at * 8];
#pragma unroll
          for (int i = 0; i < kTiles; ++i) few_mma<WT, BL>(av[u][i], sa[i], bv, sb, acc[i][b]);
        }
      }
    };
    // The loads stay ahead of the products; not pinned for float32 (2 % slower at
    // 8 and 64 tokens on 16 experts of 1024 x 4096), and for 4-bit weights with
    // eight groups, which leave no registers for two steps (48 and 81 would spill).
    constexpr bool kAhead = WT == kBf16 || (WT == kMx4 && NB < 8);
#pragma unroll 1
    for (int p = c0; p < end; p += 2 * U) {
      // what comes next: this chunk, the next one, or the next item (none: nothing)
      const bool here = p + 2 * U < end, mine = here || on;
      const uint32_t row = mine ? t.row : next.row;
      const int q = here ? t.p0 + p + 2 * U : (on ? t.p0 + c0 + chunk : next.p0);
      const int q1 = here ? t.p0 + end : (on ? t.p0 + min(len, c0 + 2 * chunk) : (more ? next.c1 : 0));
      const uint8_t* ws = m.wscale[w][st.slot] + lane_scale;
      if constexpr (WT == kMx4) {
        load_order();
        wait_vmcnt<U * kTiles>();   // this pair's scales (older than the step of weights in flight) have landed
        load_order();
        few_load_scales(a, mine ? t.s : next.s, row, q, q1, (lds_ptr)m.wscale[w][st.slot ^ 1]);
        st.slot ^= 1;
      }
      u32x4 bv[U][kTiles];
      few_load<WT, U>(a, t.w, t.row, t.p0 + p + U, t.p0 + end, bv);
      if constexpr (kAhead) load_order();
      multiply(av, p, ws);
      few_load<WT, U>(a, mine ? t.w : next.w, row, q, q1, av);
      if constexpr (kAhead) load_order();
      multiply(bv, p + U, ws + 128 * U);
      st.behind = true;
    }
    // (the last chunk's half stays the current one if the next item uses it too)
    if (c0 + chunk < span || (more && st.whole != next.rank)) st.half ^= 1;
  }
  // a wave without pieces has not fetched the next item's yet
  if (t.p1 == t.p0) {
    if constexpr (WT == kMx4) {
      st.slot ^= 1;
      few_load_scales(a, next.s, next.row, next.p0, more ? next.c1 : 0, (lds_ptr)m.wscale[w][st.slot]);
    }
    few_load<WT, U>(a, next.w, next.row, next.p0, more ? next.c1 : 0, av);
    st.behind = true;
  }
  // D[r][c] (lanes 0-7 and 16-23) + D[r + 8][c + 8] (40 lanes further) of every
  // wave, then the parts of K in order
  const int rows = kTiles * 8 * (kFewWaves >> __builtin_ctz(a.split));
  lds_barrier();   // (every wave is done with the previous item's sums)
#pragma unroll
  for (int i = 0; i < kTiles; ++i)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float other = __shfl(acc[i][b][v], (lane + 40) & 63, 64);
        if ((lane & 8) == 0 && lane < 32)
          m.red[((part * NB + b) * 8 + lr) * rows + (w >> __builtin_ctz(a.split)) * (8 * kTiles) + 8 * i + 4 * (lane >> 4) + v] =
              acc[i][b][v] + other;
      }
  lds_barrier();
  constexpr int V = kFewValues<WT, SECOND>;
  const int n0 = t.group * rows, units_log2 = __builtin_ctz(rows) - __builtin_ctz(V);
  const int stride = NB * 8 * rows;
#pragma unroll 1
  for (int o = tid; o < t.n << units_log2; o += kFewThreads) {
    const int tok = o >> units_log2, col = (o & ((1 << units_log2) - 1)) * V, n = n0 + col;
    const bool valid = n < a.N;
    float z[V];
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] = 0.f;
    for (int q = 0; q < a.split; ++q)
#pragma unroll
      for (int i = 0; i < V; ++i) z[i] += m.red[q * stride + tok * rows + col + i];
    const int s = m.l.slot[t.first + tok];
    if constexpr (SECOND) {
      // read by whichever block adds this group's experts, maybe on another XCD
      const float g = a.topk_gate[s];
      const uint64_t v = static_cast<uint64_t>(__float_as_uint(z[1] * g)) << 32 | __float_as_uint(z[0] * g);
      if (valid)
        __hip_atomic_store(reinterpret_cast<uint64_t*>(a.part + static_cast<size_t>(s) * a.N + n), v,
                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    } else {
      few_store_hidden<WT>(a, act, s, n, valid, z);
    }
  }
}

// The products of a step: persistent blocks, each with a run of neighbouring
// items.  Bound by the stream of weights: 64 tokens on 8 experts of 4096 x 11008
// (bf16, 0.72 GB a product) 135 us, 5.3 TB/s, and 151 us, 4.8 TB/s; 32 tokens on
// 32 experts of 2048 x 8192 (4 bits, 0.25 GB) 56 and 60 us, 4.4 and 4.1 TB/s.  With
// more columns an expert 4-bit weights are bound by the terms' LDS reads and
// products, and by chunks of one or a few pieces: 64 tokens on 8 experts of 4096 x
// 11008 (0.19 GB) 54 and 69 us for k = 1, 129 and 195 us for k = 2.
template <int WT, int NBMAX, bool SECOND>
__global__ __launch_bounds__(kFewThreads, NBMAX == 1 ? 4 : 2) void few_product_kernel(const FewArgs a, int act) {
  __shared__ FewLds<NBMAX> m;
  constexpr int U = 8 / kTiles;
  const int rows = kTiles * 8 * (kFewWaves >> __builtin_ctz(a.split));
  if (threadIdx.x < 64) few_lists(a.topk_idx, a.T * a.k, m.l);
  if constexpr (WT != kMx4) {
    using S = FewLds<NBMAX>;
    for (int i = threadIdx.x * 16; i < S::ZEROS; i += kFewThreads * 16)
      *reinterpret_cast<u32x4*>(reinterpret_cast<uint8_t*>(&m) + S::ZEROS_AT + i) = u32x4{0, 0, 0, 0};
  }
  __syncthreads();
  // contiguous items a block, neighbouring blocks of an XCD on neighbouring items
  const int used = __builtin_amdgcn_readfirstlane(m.l.used);
  const int items = used * a.groups, vb = xcd_virtual_block();
  const float share = static_cast<float>(items) * a.per_block;
  int item = __builtin_amdgcn_readfirstlane(static_cast<int>(static_cast<float>(vb) * share));
  const int end = vb + 1 == static_cast<int>(gridDim.x)
                      ? items
                      : __builtin_amdgcn_readfirstlane(min(items, static_cast<int>(static_cast<float>(vb + 1) * share)));
  if (item >= end) return;
  u32x4 av[U][kTiles];
  const int begin = item;
  FewItem t = few_item<WT, NBMAX, SECOND>(a, m.l, item);
  FewStage st = {0, -1, true, 0};
  few_stage_first<WT, NBMAX, SECOND>(a, m, t, 0);
  if constexpr (WT == kMx4) {
    using lds_ptr = __attribute__((address_space(3))) uint8_t*;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    few_load_scales(a, t.s, t.row, t.p0, t.c1, (lds_ptr)m.wscale[w][0]);
  }
  few_load<WT, U>(a, t.w, t.row, t.p0, t.c1, av);
#pragma unroll 1
  for (; item < end; ++item) {
    const bool more = item + 1 < end;
    const FewItem next = few_item<WT, NBMAX, SECOND>(a, m.l, more ? item + 1 : item);
    if (NBMAX == 1 || t.n <= 8) few_run<WT, 1, NBMAX, SECOND>(a, m, t, next, more, act, st, av);
    else if (t.n <= 16) few_run<WT, (NBMAX > 1 ? 2 : 1), NBMAX, SECOND>(a, m, t, next, more, act, st, av);
    else if (t.n <= 32) few_run<WT, (NBMAX > 1 ? 4 : 1), NBMAX, SECOND>(a, m, t, next, more, act, st, av);
    else few_run<WT, (NBMAX > 1 ? 8 : 1), NBMAX, SECOND>(a, m, t, next, more, act, st, av);
    t = next;
  }
  if constexpr (SECOND) {
    // Partial results are stored past the caches (agent scope), every wave waits
    // until its own have arrived, then the block counts its items done, one
    // thread an item; it adds the experts of every row group whose last item it
    // had, reading past the caches.  No cache has to be written back or emptied
    // for that: a release for each item took 79 us in place of 51 of a second
    // product of 1024 blocks.
    if (threadIdx.x == 0) m.ready = 0;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    for (int i0 = begin; i0 < end; i0 += kFewThreads) {
      const int i = i0 + static_cast<int>(threadIdx.x);
      if (i < end) {
        const int g = i % a.groups;
        if (__hip_atomic_fetch_add(a.done + g, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == used - 1)
          m.group[atomicAdd(&m.ready, 1)] = g;
      }
      __syncthreads();
      const int ready = m.ready;
      for (int o = threadIdx.x; o < ready * a.T * (rows / 4); o += kFewThreads) {
        const int col = (o & (rows / 4 - 1)) * 4, u = o >> (__builtin_ctz(rows) - 2), tok = u % a.T;
        const int n = m.group[u / a.T] * rows + col;
        if (n >= a.N) continue;
        uint64_t p[2][2] = {{0, 0}, {0, 0}};
        const uint64_t* src = reinterpret_cast<const uint64_t*>(a.part + static_cast<size_t>(tok * a.k) * a.N + n);
#pragma unroll
        for (int j = 0; j < 2; ++j)
          if (j < a.k)
#pragma unroll
            for (int q = 0; q < 2; ++q)
              p[j][q] = __hip_atomic_load(src + j * (a.N / 2) + q, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
          v[q] = __uint_as_float(static_cast<uint32_t>(p[0][q >> 1] >> (32 * (q & 1)))) +
                 __uint_as_float(static_cast<uint32_t>(p[1][q >> 1] >> (32 * (q & 1))));
        if constexpr (WT == kF32) {
          *reinterpret_cast<float4*>(static_cast<float*>(a.y) + static_cast<size_t>(tok) * a.N + n) =
              make_float4(v[0], v[1], v[2], v[3]);
        } else {
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.y) + static_cast<size_t>(tok) * a.N + n) =
              make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        }
      }
      __syncthreads();
      if (threadIdx.x == 0) m.ready = 0;
      __syncthreads();
    }
  }
}

// Up to eight slots (tokens times choices): the same products and sums, bit for
// bit, with nothing before the first load of weights that can be left out.  With
// so few columns latency is all there is, so a block has one item (second
// product: the same rows of every expert, one after the other, so that it can
// add a token's experts itself), its columns come straight into registers, and
// no list is built: lane s knows slot s's expert and which slots share it.
// Seven tokens on 4 experts of 256 x 1024 (float32): 13.4 and 16.3 us by the
// kernel above, 8.8 and 10.3 here; one token on two of 1024 x 4096 (bf16): 12.8
// and 15.3, 10.2 and 13.2; on one of 4096 x 11008 (4 bits), second: 19.8, 15.4.
template <int WT, int RT, bool SECOND>
struct DirectStep {
  static constexpr int BL = FewLayout<WT, SECOND>::BL, U = BL == 1 ? 4 : (BL <= 4 ? 2 : 1);   // pieces of K
  u32x4 w[U][RT], col[U][BL];
  int sw[U][RT], sc[U];
};

template <int WT, int RT, bool SECOND>
__global__ __launch_bounds__(SECOND ? 2 * kFewThreads : kFewThreads, 4) void few_direct_kernel(const FewArgs a, int act) {
  using Step = DirectStep<WT, RT, SECOND>;
  constexpr int U = Step::U, BL = Step::BL, V = kFewValues<WT, SECOND>;
  __shared__ float red[kDirectSlots * 8 * RT * kFewWaves];   // [part][slot][row]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int w = wave % kFewWaves;
  const int slots = a.T * a.k, lr = lane & 7, lc = lane >> 3;
  const int es = lane < slots ? a.topk_idx[lane] : -1;
  uint32_t same = 0;
#pragma unroll
  for (int j = 0; j < kDirectSlots; ++j) {
    const uint32_t m = static_cast<uint32_t>(__ballot(lane < slots && es == __builtin_amdgcn_readlane(es, j)));
    if (lane == j) same = m;
  }
  // the first slot of every expert in use
  uint32_t todo = static_cast<uint32_t>(__ballot(lane < slots && __builtin_ctz(same | 1u << 31) == lane));
  int group = blockIdx.x;
  if constexpr (!SECOND) {
    const int rank = blockIdx.x / a.groups;
    group -= rank * a.groups;
    for (int r = 0; r < rank; ++r) todo &= todo - 1;
    if (todo == 0) return;
    todo &= -todo;
  }
  const int kbytes = few_kbytes<WT>(a.K), pieces = (kbytes + 127) / 128, split_log2 = __builtin_ctz(a.split);
  const int part = w & (a.split - 1), rows = 8 * RT * kFewWaves >> split_log2, in_block = (w >> split_log2) * (8 * RT);
  const uint32_t row = group * rows + in_block;
  const int p0 = (part * pieces) >> split_log2;
  const int p1 = static_cast<int>(row) < a.N ? ((part + 1) * pieces) >> split_log2 : p0;
  const int steps = (((pieces + a.split - 1) >> split_log2) + U - 1) / U;   // of the longest part
  const int pitch = few_pitch<WT, SECOND>(a.K), scale_pitch = few_scale_pitch(a.K);
  const __amdgpu_buffer_rsrc_t in = few_rsrc(a.in), ins = few_rsrc(WT == kMx4 ? a.in_scale : a.in);
  // the slot of this lane's column under a mask of slots (those past the last
  // repeat it; their products are not used)
  auto slot_of = [&](uint32_t mask) {
    for (int i = 0; i < lr; ++i)
      if (mask & (mask - 1)) mask &= mask - 1;
    return __builtin_ctz(mask);
  };
  // what does not exist is not fetched and reads as zeros
  auto load = [&](int e, uint32_t mask, int step, bool on, Step& s) {
    const __amdgpu_buffer_rsrc_t wr = few_rsrc(a.w + static_cast<size_t>(e) * a.N * kbytes);
    const int slot = slot_of(mask);
    const uint32_t column = SECOND || a.k == 1 ? slot : slot >> 1;
    const int first = p0 + step * U;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int p = first + u;
      const bool here = on && p < p1 && p * 128 + 16 * lc < kbytes;
#pragma unroll
      for (int i = 0; i < RT; ++i)
        s.w[u][i] = __builtin_amdgcn_raw_buffer_load_b128(
            wr, here ? (row + 8 * i + lr) * kbytes + p * 128 + 16 * lc : kFewRange, 0, 2);
    }
    if constexpr (WT == kMx4) {
      const __amdgpu_buffer_rsrc_t sr = few_rsrc(a.w_scale + static_cast<size_t>(e) * pieces * a.N * 8);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int p = first + u;
        const bool here = on && p < p1;
#pragma unroll
        for (int i = 0; i < RT; ++i)
          s.sw[u][i] = __builtin_amdgcn_raw_buffer_load_b8(
              sr, here ? (p * a.N + row + 8 * i + lr) * 8 + lc : kFewRange, 0, 0);
        s.sc[u] = __builtin_amdgcn_raw_buffer_load_b8(ins, here ? column * scale_pitch + p * 8 + lc : kFewRange, 0, 0);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int p = first + u;
#pragma unroll
      for (int j = 0; j < BL; ++j)
        s.col[u][j] = __builtin_amdgcn_raw_buffer_load_b128(
            in, on && p < p1 ? column * pitch + (p * BL + j) * 128 + 16 * lc : kFewRange, 0, 0);
    }
  };
  // second product: a block of 16 waves takes two experts at a time
  const int teams = SECOND ? blockDim.x / kFewThreads : 1;
  if (SECOND && wave >= kFewWaves) todo &= todo - 1;
  int step = 0, first = todo ? __builtin_ctz(todo) : 0;
  uint32_t mask = __builtin_amdgcn_readlane(same, first);
  Step cur;
  load(__builtin_amdgcn_readlane(es, first), mask, 0, todo != 0, cur);
  f32x4 acc[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  while (todo) {
    const uint32_t at = mask;
    const bool last = ++step == steps;   // of this expert
    if (last) {
      step = 0;
      todo &= todo - 1;
      if (teams > 1) todo &= todo - 1;
    }
    const bool more = todo != 0;
    if (more) first = __builtin_ctz(todo);
    mask = __builtin_amdgcn_readlane(same, first);
    Step next;
    load(__builtin_amdgcn_readlane(es, first), mask, step, more, next);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < RT; ++i)
        few_mma<WT, BL>(cur.w[u][i], WT == kMx4 ? cur.sw[u][i] : 0, cur.col[u], WT == kMx4 ? cur.sc[u] : 0, acc[i]);
    if (last) {
      const int slot = slot_of(at), n = __builtin_popcount(at);
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float other = __shfl(acc[i][v], (lane + 40) & 63, 64);
          if ((lane & 8) == 0 && lane < 32 && lr < n)
            red[(part * kDirectSlots + slot) * rows + in_block + 8 * i + 4 * (lane >> 4) + v] = acc[i][v] + other;
          acc[i][v] = 0.f;
        }
    }
    cur = next;
  }
  __syncthreads();
  const int units = rows / V;
  auto sums = [&](int slot, int col, float (&z)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] = 0.f;
    for (int q = 0; q < a.split; ++q)
#pragma unroll
      for (int i = 0; i < V; ++i) z[i] += red[(q * kDirectSlots + slot) * rows + col + i];
  };
  for (int o = tid; o < (SECOND ? a.T : slots) * units; o += blockDim.x) {
    const int s = o / units, col = (o - s * units) * V, n = group * rows + col;
    const bool valid = n < a.N;
    if constexpr (SECOND) {
#pragma clang fp contract(off)   // each expert's part is rounded, as where they are added from memory
      float y[V];
#pragma unroll
      for (int i = 0; i < V; ++i) y[i] = 0.f;
      for (int j = 0; j < a.k; ++j) {
        float z[V];
        sums(s * a.k + j, col, z);
        const float g = a.topk_gate[s * a.k + j];
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = j == 0 ? z[i] * g : y[i] + z[i] * g;
      }
      if (!valid) continue;
      if constexpr (WT == kF32)
        *reinterpret_cast<float2*>(static_cast<float*>(a.y) + static_cast<size_t>(s) * a.N + n) = make_float2(y[0], y[1]);
      else
        *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.y) + static_cast<size_t>(s) * a.N + n) =
            pack_bf16x2(y[0], y[1]);
    } else {
      if (!(mask >> s & 1)) continue;
      float z[V];
      sums(s, col, z);
      few_store_hidden<WT>(a, act, s, n, valid, z);
    }
  }
}

struct FewWs {
  FewTerms f;
  uint8_t* h;      // hidden rows
  float* part;
  int* done;
};

// one layout serves every weight type: 4 bytes a hidden value (4-bit weights: 3
// and the scales)
FewWs carve_few(Carver& c, int T, int d, int k, int d_ff) {
  const size_t slots = static_cast<size_t>(T) * k;
  FewWs w;
  w.f.x8 = c.take<uint8_t>(static_cast<size_t>(T) * few_pitch<kMx4, false>(d));
  w.f.x8_scale = c.take<uint8_t>(static_cast<size_t>(T) * few_scale_pitch(d));
  w.h = c.take<uint8_t>(slots * align_up(d_ff, 256) * 4);
  w.f.h8 = w.h;
  w.f.h8_scale = c.take<uint8_t>(slots * few_scale_pitch(d_ff));
  w.f.d_ff = d_ff;
  w.part = c.take<float>(slots * d);
  w.done = c.take<int>(d / 8);
  return w;
}

template <int WT, int NBMAX, bool SECOND>
void launch_few_nb(FewArgs a, int act, hipStream_t s) {
  // most parts of K whose columns (an expert has at most T) fit the buffer
  while (a.split > 1 && few_chunk<WT, SECOND, NBMAX>(__builtin_ctz(a.split), few_cols_log2(a.T)) < 1) a.split /= 2;
  const int grid = persistent_grid() * (NBMAX == 1 ? 2 : 1);
  const int rows = 8 * kTiles * kFewWaves / a.split;
  a.groups = (a.N + rows - 1) / rows;
  a.per_group = 1.0f / a.groups;
  a.per_block = 1.0f / grid;
  launch(SECOND ? "few_ffn2" : "few_ffn1", few_product_kernel<WT, NBMAX, SECOND>, grid, kFewThreads, 0, s, a, act);
}

// Rows of an item.  More rows take their columns to LDS less often; fewer give
// every CU an item and split K over more waves.  So: the fewest parts of K with
// an item a CU, and eight where no number of parts gives that.  61 tokens on 16
// experts of 1024 x 4096 (bf16), second product: 1, 2 and 4 parts (128, 256,
// 512 items) 48, 41 and 40 us; 64 tokens on 8 experts of 4096 x 11008: 1 and 2
// parts (256, 512 items) 141 and 151 us; one token on two experts of 1024 x
// 4096: 1, 2, 4 and 8 parts (16 to 128 items) 62, 35, 24 and 16 us.
template <int WT, bool SECOND>
void launch_few(FewArgs a, int E, int act, hipStream_t s) {
  // experts in use, expected at an even load
  double idle = 1.0;
  for (int t = 0; t < a.T; ++t) idle *= 1.0 - static_cast<double>(a.k) / E;
  const double used = std::max(1.0, E * (1.0 - idle));
  constexpr int kRows = 8 * 2 * kFewWaves;
  a.split = 1;
  while (a.split < kFewWaves && used * ((a.N * a.split + kRows - 1) / kRows) < persistent_grid()) a.split *= 2;
  if (WT == kMx4 && !SECOND) a.split = std::min(a.split, 4);   // whole blocks of 32 hidden values
  // Without LDS columns: up to two slots, or eight on experts of 32 MB together
  // (the second product takes a block's experts one after the other).  Whole
  // calls, us, few_product_kernel | few_direct_kernel: bf16, 1024 x 4096 of 16,
  // k = 2, one token 29.1 | 25.2, two 32.4 | 32.0, four (56 MB) 37.6 | 45.3; 4096
  // x 11008 of 8, k = 2, three tokens 191 | 250; float32, 256 x 1024 of 4, seven
  // tokens 28.6 | 20.7, 1024 x 1024 of 4, eight (17 MB) 32.2 | 22.3.
  // (4-bit tokens, four units a piece: 17.9 us against 14.9 through LDS for one
  // token of 4096 -> 11008)
  const int slots = a.T * a.k;
  bool direct = slots <= 2 || (slots <= kDirectSlots && used * a.N * few_kbytes<WT>(a.K) <= 32e6);
  if constexpr (WT == kMx4 && !SECOND) direct = false;
  else if (direct) {
    // half the rows a wave where a block a CU needs it
    const int experts = SECOND ? 1 : std::min(slots, E), threads = SECOND && slots > 1 ? 2 * kFewThreads : kFewThreads;
    const bool half = static_cast<long long>(a.N) * a.split * experts < static_cast<long long>(kRows) * persistent_grid();
    const int rows = (half ? kRows / 2 : kRows) / a.split;
    a.groups = (a.N + rows - 1) / rows;
    launch(SECOND ? "few_ffn2" : "few_ffn1", half ? few_direct_kernel<WT, 1, SECOND> : few_direct_kernel<WT, 2, SECOND>,
           a.groups * experts, threads, 0, s, a, act);
  }
  if (direct) return;
  if (a.T <= 8) launch_few_nb<WT, 1, SECOND>(a, act, s);
  else launch_few_nb<WT, 8, SECOND>(a, act, s);
}

template <int WT>
void run_few(const void* x, int T, int d, const void* w_gate, const float* b_gate, int E, int k, const void* w1,
             const void* s1, const void* w2, const void* s2, int d_ff, int act, int32_t* topk_idx,
             float* topk_gate, void* y, const FewWs& ws, hipStream_t s) {
  FewTerms f = ws.f;
  if (WT != kMx4) f.x8 = nullptr;
  launch("few_gate", few_gate_kernel<WT == kF32>, T, kGateThreads, 0, s, x, d, w_gate, b_gate, E, k, topk_idx,
         topk_gate, f, ws.done, d / 8);
  FewArgs a = {};
  a.T = T;
  a.k = k;
  a.topk_idx = topk_idx;
  a.topk_gate = topk_gate;
  a.w = static_cast<const uint8_t*>(w1);
  a.w_scale = static_cast<const uint8_t*>(s1);
  a.in = WT == kMx4 ? ws.f.x8 : static_cast<const uint8_t*>(x);
  a.in_scale = ws.f.x8_scale;
  a.N = d_ff;
  a.K = d;
  a.h = ws.h;
  a.h_scale = ws.f.h8_scale;
  launch_few<WT, false>(a, E, act, s);
  a.w = static_cast<const uint8_t*>(w2);
  a.w_scale = static_cast<const uint8_t*>(s2);
  a.in = ws.h;
  a.in_scale = ws.f.h8_scale;
  a.N = d;
  a.K = d_ff;
  a.part = ws.part;
  a.done = ws.done;
  a.y = y;
  launch_few<WT, true>(a, E, act, s);
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
  if (few_misaligned(x) || few_misaligned(w_gate) || few_misaligned(w1) || few_misaligned(w2) || few_misaligned(y))
    return fail(LUFFY_E_INVALID, "luffy_moe_few: x, w_gate, w1, w2 and y must be 16-byte aligned");
  if (weight_type == LUFFY_MX4 &&
      ((reinterpret_cast<uintptr_t>(w1_scale) | reinterpret_cast<uintptr_t>(w2_scale)) & 7u) != 0)
    return fail(LUFFY_E_INVALID, "luffy_moe_few: scales must be 8-byte aligned");
  if (weight_type != LUFFY_MX4 && static_cast<long long>(d) * d_ff * elem_bytes(dtype) > 0xFFFF0000ll)
    return fail(LUFFY_E_UNSUPPORTED, "luffy_moe_few: one expert's weights exceed 4 GiB - 64 KiB");
  const size_t need = luffy_moe_few_workspace_size(T, d, E, k, d_ff);
  if (workspace_bytes < need || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return fail(LUFFY_E_WORKSPACE, "luffy_moe_few: workspace needs %zu bytes, 256-aligned", need);
  hipStream_t s = static_cast<hipStream_t>(stream);
  Carver c(workspace);
  const FewWs ws = carve_few(c, T, d, k, d_ff);
  if (weight_type == LUFFY_F32)
    run_few<kF32>(x, T, d, w_gate, b_gate, E, k, w1, w1_scale, w2, w2_scale, d_ff, act, topk_idx, topk_gate, y, ws, s);
  else if (weight_type == LUFFY_BF16)
    run_few<kBf16>(x, T, d, w_gate, b_gate, E, k, w1, w1_scale, w2, w2_scale, d_ff, act, topk_idx, topk_gate, y, ws, s);
  else
    run_few<kMx4>(x, T, d, w_gate, b_gate, E, k, w1, w1_scale, w2, w2_scale, d_ff, act, topk_idx, topk_gate, y, ws, s);
  return check_launch("luffy_moe_few");
}
