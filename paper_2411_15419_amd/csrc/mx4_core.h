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

// Keeps the loads before it (plain ones and DMA to LDS) before those after it.  A
// counted wait (all but the n newest loads of this wave have landed) is right
// only for the order it was counted on, and to the compiler plain loads and DMA
// to LDS are independent.
__device__ __forceinline__ void load_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(1);   // arithmetic may cross
}

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

  // Wave w: P rows wave_m(w) WTM.., Q blocks of 32 rows wave_n(w), wave_n(w) +
  // WN, ... (a tile with few Q rows keeps every wave equally busy: active_q).
  static __device__ __forceinline__ int wave_m(int w) { return w % WM; }
  static __device__ __forceinline__ int wave_n(int w) { return w / WM; }
  static __device__ __forceinline__ int q_row(int wn, int fn) { return 32 * (wn + WN * fn); }
  static __device__ __forceinline__ int active_q(int wn, int rows) {
    return min(max((rows - 32 * wn + 32 * WN - 1) / (32 * WN), 0), FN);
  }

  struct Frags {
    i32x4 a[FM], b[FN];
  };
  struct Scales {
    int a[FM], b[FN];
  };
  struct Addr {
    int prow, qrow, half, sw, ps, qs;   // fragment rows and scales in a stage
  };
  static __device__ __forceinline__ Addr addr(int wm, int wn) {
    const int lane = opaque_tid() & 63;
    Addr a;
    a.half = lane >> 5;
    a.sw = swz(lane & 31);
    a.prow = (wm * WTM + (lane & 31)) * 128;
    a.qrow = BM * 128 + (32 * wn + (lane & 31)) * 128;
    a.ps = SCALE_AT + (wm * WTM + (lane & 31)) * 8 + 4 * a.half;
    a.qs = SCALE_Q_AT + (32 * wn + (lane & 31)) * 8 + 4 * a.half;
    return a;
  }
  // fragments of step `step` of the stage at st, first NQ Q blocks
  template <int NQ>
  static __device__ __forceinline__ void read_step(lds_ptr st, const Addr& ad, int step, Frags& f) {
    const int at = ((4 * ad.half + step) ^ ad.sw) * 16;
#pragma unroll
    for (int i = 0; i < FM; ++i)
      f.a[i] = *reinterpret_cast<const __attribute__((address_space(3))) i32x4*>(st + ad.prow + 32 * i * 128 + at);
#pragma unroll
    for (int j = 0; j < NQ; ++j)
      f.b[j] = *reinterpret_cast<const __attribute__((address_space(3))) i32x4*>(st + ad.qrow + 32 * WN * j * 128 + at);
  }
  template <int NQ>
  static __device__ __forceinline__ void read_scales(lds_ptr st, const Addr& ad, Scales& s) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
      s.a[i] = *reinterpret_cast<const __attribute__((address_space(3))) int*>(st + ad.ps + 32 * i * 8);
#pragma unroll
    for (int j = 0; j < NQ; ++j)
      s.b[j] = *reinterpret_cast<const __attribute__((address_space(3))) int*>(st + ad.qs + 32 * WN * j * 8);
  }
  template <int NQ, int STEP>
  static __device__ __forceinline__ void mma_step(const Frags& f, const Scales& s, Acc& acc) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < NQ; ++j) acc[i][j] = mfma32x32x64_f4<STEP>(f.a[i], f.b[j], acc[i][j], s.a[i], s.b[j]);
  }

  // Instruction order of a step: the next step's LDS reads two after an MFMA
  // from the first on, so they have landed when the next step starts.
  template <int NQ>
  static __device__ __forceinline__ void interleave_reads() {
    constexpr int NMF = FM * NQ, NDS = FM + NQ;
#pragma unroll
    for (int i = 0; i < NMF; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // MFMA
      if (2 * i + 1 < NDS) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);   // DS read
      else if (2 * i < NDS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    if constexpr (NDS > 2 * NMF) __builtin_amdgcn_sched_group_barrier(0x100, NDS - 2 * NMF, 0);
  }
  // The step after the barrier: the next stage's DMA goes out first, one after
  // an MFMA; then the reads (fragments and scales).
  template <int NQ>
  static __device__ __forceinline__ void interleave_loads() {
    constexpr int NMF = FM * NQ, NDS = 2 * (FM + NQ);
    constexpr int PV = NMF < LOADS ? NMF : LOADS;
#pragma unroll
    for (int i = 0; i < PV; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // MFMA
      __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);   // VMEM read
    }
    if constexpr (NMF > PV) __builtin_amdgcn_sched_group_barrier(0x008, NMF - PV, 0);
    if constexpr (LOADS > PV) __builtin_amdgcn_sched_group_barrier(0x020, LOADS - PV, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, NDS, 0);
  }

  // waits until at most min(n, 1) stages of this wave's DMA are outstanding
  static __device__ __forceinline__ void wait_stages(int n) {
    if (n >= 1) wait_vmcnt<LOADS>();
    else wait_vmcnt<0>();
  }

  template <int NQ>
  static __device__ __forceinline__ void stage_steps(lds_ptr cur, const Addr& ad, const Scales& sc, Frags (&f)[2],
                                                     Acc& acc, bool sched) {
    if (sched) __builtin_amdgcn_sched_barrier(0);
    read_step<NQ>(cur, ad, 1, f[1]);
    mma_step<NQ, 0>(f[0], sc, acc);
    if (sched) interleave_reads<NQ>();
    if (sched) __builtin_amdgcn_sched_barrier(0);
    read_step<NQ>(cur, ad, 2, f[0]);
    mma_step<NQ, 1>(f[1], sc, acc);
    if (sched) interleave_reads<NQ>();
    if (sched) __builtin_amdgcn_sched_barrier(0);
    read_step<NQ>(cur, ad, 3, f[1]);
    mma_step<NQ, 2>(f[0], sc, acc);
    if (sched) interleave_reads<NQ>();
  }

  // Issues stages FROM .. TO - 1 of a tile (of its first STAGES; FROM = 0 first).
  template <int FROM, int TO>
  static __device__ __forceinline__ void prefetch(const Tile& t, Pipe& s, uint8_t* lds_generic) {
    const lds_ptr lds = (lds_ptr)lds_generic;
    if constexpr (FROM == 0) setup(t, s);
    const int nk = __builtin_amdgcn_readfirstlane((t.kbytes + 127) / 128);
#pragma unroll
    for (int k = FROM; k < TO; ++k) {
      if (k < nk) issue(t, s, k, lds + k * STAGE_BYTES);
      load_order();
    }
  }

  // The product of a tile whose first stages are on their way; the wave
  // multiplies its first NQ Q blocks, but takes part in every load and barrier.
  // Result layout: acc[i][j][v] of lane l of wave w is P row wave_m(w) WTM +
  // 32 i + 8 (v / 4) + 4 (l / 32) + v % 4 and Q row q_row(wave_n(w), j) +
  // l % 32.  Ends with a barrier after which the LDS may be used again.
  //
  // Fragments are double-buffered a step: while the MFMAs of step s run, step
  // s + 1 is read; after the last read of a stage every wave waits for the next
  // stage's DMA, one barrier frees the stage's buffer, and the DMA of the stage
  // after the ring goes into it under the last step's MFMAs.
  template <int NQ>
  static __device__ __forceinline__ void run(const Tile& t, const Pipe& s, uint8_t* lds_generic, Acc& acc) {
    const lds_ptr lds = (lds_ptr)lds_generic;
    const int w = wave();
    const int nk = __builtin_amdgcn_readfirstlane((t.kbytes + 127) / 128);
    wait_stages(min(nk, STAGES) - 1);
    raw_barrier();
    const Addr ad = addr(wave_m(w), wave_n(w));
    Frags f[2];
    Scales sc;
    read_scales<NQ>(lds, ad, sc);
    read_step<NQ>(lds, ad, 0, f[0]);
    int kt = 0, cb = 0;
    // steady state: stage kt + STAGES exists
    for (; kt + STAGES < nk; ++kt) {
      const lds_ptr cur = lds + cb * STAGE_BYTES;
      cb = cb + 1 == STAGES ? 0 : cb + 1;
      const lds_ptr nxt = lds + cb * STAGE_BYTES;
      stage_steps<NQ>(cur, ad, sc, f, acc, true);
      __builtin_amdgcn_sched_barrier(0);
      wait_vmcnt<(STAGES - 2) * LOADS>();   // stage kt + 1 has landed (this wave's part)
      __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): own reads of stage kt are done
      raw_barrier();
      __builtin_amdgcn_sched_barrier(0);
      issue(t, s, kt + STAGES, cur);
      Scales ns;
      read_scales<NQ>(nxt, ad, ns);
      read_step<NQ>(nxt, ad, 0, f[0]);
      mma_step<NQ, 3>(f[1], sc, acc);
      interleave_loads<NQ>();
      __builtin_amdgcn_sched_barrier(0);
      sc = ns;
    }
    for (; kt < nk; ++kt) {
      const lds_ptr cur = lds + cb * STAGE_BYTES;
      cb = cb + 1 == STAGES ? 0 : cb + 1;
      stage_steps<NQ>(cur, ad, sc, f, acc, false);
      Scales ns = sc;
      if (kt + 1 < nk) {
        wait_stages(nk - 2 - kt);
        __builtin_amdgcn_s_waitcnt(0xC07F);
        raw_barrier();
        read_scales<NQ>(lds + cb * STAGE_BYTES, ad, ns);
        read_step<NQ>(lds + cb * STAGE_BYTES, ad, 0, f[0]);
      }
      mma_step<NQ, 3>(f[1], sc, acc);
      sc = ns;
    }
    __syncthreads();
  }

  static __device__ __forceinline__ void zero(Acc& acc) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
  }

  // prefetch() and run() with the number of Q blocks that hold a valid row
  // (a wave without one: no MFMAs).
  template <int N = FN>
  static __device__ __forceinline__ void run_nq(int nq, const Tile& t, const Pipe& s, uint8_t* lds, Acc& acc) {
    if constexpr (N == 0) {
      run<0>(t, s, lds, acc);
    } else {
      if (nq >= N) run<N>(t, s, lds, acc);
      else run_nq<N - 1>(nq, t, s, lds, acc);
    }
  }
};

}  // namespace luffy
