// Tile core of the microscaled 4-bit product on gfx950's block-scaled MFMA:
// C[i][j] = sum_k P[i][k] Q[j][k], P and Q rows of 4-bit values (two a byte, K
// contiguous) with a scale byte per 32 values (stored [K / 256][row][8]).
//
// A stage holds 256 values of K: 128 bytes of every row, fetched straight into
// LDS eight rows a DMA instruction, the row's eight 16-byte blocks permuted by
// (row >> 1) & 7 so that fragment reads fall on distinct banks, and the rows'
// eight scale bytes.  v_mfma_scale_f32_32x32x64_f8f6f4 takes one block of 32
// values a lane with its scale byte picked out of a register by an immediate:
// lanes 0-31 take blocks 0-3 of the stage in its four steps and lanes 32-63
// blocks 4-7 (the sum over K may pair any two blocks), so that a row's scales
// of one stage are one 4-byte LDS read a lane.
#pragma once

#include "gemm_core.h"

namespace luffy {

typedef int i32x4 __attribute__((ext_vector_type(4)));

template <int STEP>
__device__ __forceinline__ f32x16 mfma32x32x64_f4(i32x4 a, i32x4 b, f32x16 c, int sa, int sb) {
  const i32x8 av = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
  const i32x8 bv = __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1);
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(av, bv, c, 4, 4, STEP, sa, STEP, sb);
}

// Block exponent (biased by 127) of values whose largest absolute value has
// the float32 bits `most`: floor(log2 most) - 2, at least -127; 255 for an
// infinity or a NaN.
__device__ __forceinline__ uint32_t mx4_exponent(uint32_t most) {
  const uint32_t ex = most >> 23;
  return ex == 255u ? 255u : (ex > 2u ? ex - 2u : 0u);
}

template <int BM_, int BN_, int WM_, int WN_, int STAGES_>
struct Mx4Core {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_;
  static constexpr int NWAVES = WM * WN, THREADS = 64 * NWAVES;
  static constexpr int WTM = BM / WM, WTN = BN / WN, FM = WTM / 32, FN = WTN / 32;
  static constexpr int kStageK = 256;                          // values of K a stage
  static constexpr int LP = BM / 8 / NWAVES, LQ = BN / 8 / NWAVES;   // data DMA instructions a wave and stage
  static constexpr int SP = (BM / 32 + NWAVES - 1) / NWAVES, SQ = (BN / 32 + NWAVES - 1) / NWAVES;   // scales
  static constexpr int LOADS = LP + LQ + SP + SQ;
  static constexpr int SCALE_AT = (BM + BN) * 128;
  static constexpr int SCALE_Q_AT = SCALE_AT + SP * NWAVES * 256;
  static constexpr int STAGE_BYTES = SCALE_Q_AT + SQ * NWAVES * 256;
  static constexpr int LDS_BYTES = STAGES * STAGE_BYTES;
  static_assert(LP * NWAVES * 8 == BM && LQ * NWAVES * 8 == BN, "load plan");
  static_assert(STAGES >= 2 && (STAGES - 1) * LOADS < 64 && LDS_BYTES <= 160 * 1024, "ring");

  using Acc = f32x16[FM][FN];
  using lds_ptr = __attribute__((address_space(3))) uint8_t*;
  using Rsrc = __amdgpu_buffer_rsrc_t;
  static constexpr uint32_t kRange = 0xFFFF0000u;

  static __device__ __forceinline__ Rsrc rsrc(const uint8_t* base) {
    const uint64_t v = reinterpret_cast<uint64_t>(base);
    const uint64_t lo = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v)));
    const uint64_t hi = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v >> 32)));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((hi << 32) | lo), static_cast<short>(0),
                                             static_cast<int>(kRange), 0x00020000);
  }
  static __device__ __forceinline__ void dma(Rsrc r, lds_ptr dst, uint32_t off, int soff, bool wide) {
    if (wide)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, reinterpret_cast<__attribute__((address_space(3))) void*>(dst), 16,
                                               off, soff, 0, 0);
    else
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, reinterpret_cast<__attribute__((address_space(3))) void*>(dst), 4,
                                               off, soff, 0, 0);
  }

  // Operands of a tile: first row of each (values and stage 0's scales), rows
  // that exist, bytes between stages of the scales, bytes of a row.
  struct Tile {
    const uint8_t *p, *q, *ps, *qs;
    int pvalid, qvalid;
    size_t ps_stage, qs_stage;
    int kbytes;
  };
  struct Pipe {
    Rsrc p, q;
    uint32_t off[LP + LQ], soff[SP + SQ];
    int chunk;   // byte of this lane's chunk in a stage row (the same in all its loads)
  };

  static __device__ __forceinline__ int wave() { return __builtin_amdgcn_readfirstlane(opaque_tid() >> 6); }
  static __device__ __forceinline__ int swz(int r) { return (r >> 1) & 7; }

  static __device__ __forceinline__ void setup(const Tile& t, Pipe& s) {
    const int lane = opaque_tid() & 63, w = wave();
    s.p = rsrc(t.p);
    s.q = rsrc(t.q);
    // rows 8 (w + NWAVES j) + lane / 8: j moves a row by a multiple of 16, so
    // the permutation is the same in every load
    static_assert(NWAVES % 2 == 0, "chunk permutation");
    s.chunk = 16 * ((lane & 7) ^ swz(8 * w + (lane >> 3)));
#pragma unroll
    for (int j = 0; j < LP + LQ; ++j) {
      const int r = 8 * (w + NWAVES * (j < LP ? j : j - LP)) + (lane >> 3);
      s.off[j] = r < (j < LP ? t.pvalid : t.qvalid) ? static_cast<uint32_t>(r) * t.kbytes + s.chunk : kRange;
    }
#pragma unroll
    for (int j = 0; j < SP + SQ; ++j) {
      const int r = 32 * (w + NWAVES * (j < SP ? j : j - SP)) + (lane >> 1);
      s.soff[j] = r < (j < SP ? t.pvalid : t.qvalid) ? 8u * r + 4u * (lane & 1) : kRange;
    }
  }

  // DMA of stage kt into the buffer at st.  Blocks past the row's end (K no
  // multiple of 256) are not fetched: they read as zeros.
  static __device__ __forceinline__ void issue(const Tile& t, const Pipe& s, int kt, lds_ptr st) {
    const int w = wave();
    const bool in = kt * 128 + s.chunk < t.kbytes;
#pragma unroll
    for (int j = 0; j < LP + LQ; ++j) {
      const lds_ptr dst = st + (j < LP ? 0 : BM * 128) + (w + NWAVES * (j < LP ? j : j - LP)) * 1024;
      dma(j < LP ? s.p : s.q, dst, in ? s.off[j] : kRange, kt * 128, true);
    }
    const Rsrc ps = rsrc(t.ps + t.ps_stage * kt), qs = rsrc(t.qs + t.qs_stage * kt);
#pragma unroll
    for (int j = 0; j < SP + SQ; ++j) {
      const lds_ptr dst = st + (j < SP ? SCALE_AT : SCALE_Q_AT) + (w + NWAVES * (j < SP ? j : j - SP)) * 256;
      dma(j < SP ? ps : qs, dst, s.soff[j], 0, false);
    }
  }

  template <int STEP>
  static __device__ __forceinline__ void step(lds_ptr prow, lds_ptr qrow, int half, int sw, const int (&sa)[FM],
                                              const int (&sb)[FN], Acc& acc) {
    const int at = ((4 * half + STEP) ^ sw) * 16;
    i32x4 a[FM], b[FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
      a[i] = *reinterpret_cast<const __attribute__((address_space(3))) i32x4*>(prow + 32 * i * 128 + at);
#pragma unroll
    for (int j = 0; j < FN; ++j)
      b[j] = *reinterpret_cast<const __attribute__((address_space(3))) i32x4*>(qrow + 32 * j * 128 + at);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = mfma32x32x64_f4<STEP>(a[i], b[j], acc[i][j], sa[i], sb[j]);
  }

  // The whole product of a tile.  Result layout: acc[i][j][v] of lane l of wave
  // w is P row (w / WN) WTM + 32 i + 8 (v / 4) + 4 (l / 32) + v % 4 and Q row
  // (w % WN) WTN + 32 j + l % 32.  Ends with a barrier after which the LDS may
  // be used again.
  static __device__ __forceinline__ void run(const Tile& t, uint8_t* lds_generic, Acc& acc) {
    const lds_ptr lds = (lds_ptr)lds_generic;
    const int lane = opaque_tid() & 63, w = wave(), wm = w / WN, wn = w % WN;
    Pipe s;
    setup(t, s);
    const int nk = __builtin_amdgcn_readfirstlane((t.kbytes + 127) / 128);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
#pragma unroll
    for (int k = 0; k < STAGES - 1; ++k)
      if (k < nk) issue(t, s, k, lds + k * STAGE_BYTES);
    const int half = lane >> 5, sw = swz(lane & 31);
    const int prow = (wm * WTM + (lane & 31)) * 128, qrow = BM * 128 + (wn * WTN + (lane & 31)) * 128;
    const int psc = SCALE_AT + (wm * WTM + (lane & 31)) * 8 + 4 * half;
    const int qsc = SCALE_Q_AT + (wn * WTN + (lane & 31)) * 8 + 4 * half;
    int buf = 0;
    for (int kt = 0; kt < nk; ++kt) {
      // stage kt has landed (this wave's part); then every wave's, and every
      // wave is done with the buffer of stage kt - 1
      if (kt + STAGES - 2 < nk) wait_vmcnt<(STAGES - 2) * LOADS>();
      else wait_vmcnt<0>();
      __builtin_amdgcn_s_waitcnt(0xC07F);
      raw_barrier();
      const int free_buf = buf == 0 ? STAGES - 1 : buf - 1;
      if (kt + STAGES - 1 < nk) issue(t, s, kt + STAGES - 1, lds + free_buf * STAGE_BYTES);
      const lds_ptr st = lds + buf * STAGE_BYTES;
      int sa[FM], sb[FN];
#pragma unroll
      for (int i = 0; i < FM; ++i)
        sa[i] = *reinterpret_cast<const __attribute__((address_space(3))) int*>(st + psc + 32 * 8 * i);
#pragma unroll
      for (int j = 0; j < FN; ++j)
        sb[j] = *reinterpret_cast<const __attribute__((address_space(3))) int*>(st + qsc + 32 * 8 * j);
      step<0>(st + prow, st + qrow, half, sw, sa, sb, acc);
      step<1>(st + prow, st + qrow, half, sw, sa, sb, acc);
      step<2>(st + prow, st + qrow, half, sw, sa, sb, acc);
      step<3>(st + prow, st + qrow, half, sw, sa, sb, acc);
      buf = buf + 1 == STAGES ? 0 : buf + 1;
    }
    __syncthreads();
  }
};

}  // namespace luffy
