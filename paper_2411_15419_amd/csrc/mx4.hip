// Microscaled 4-bit matrices (E2M1 values in blocks of 32 with an E8M0 scale):
// luffy_mx4_quantize and luffy_mx4_dequantize, luffy_mx4_matmul and
// luffy_mx4_expert_ffn.
#include <algorithm>

#include "act.h"
#include "luffy_common.h"
#include "mx4_core.h"

namespace luffy {
namespace {

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Codes of eight consecutive values under a block's scale, four bits each.
__device__ __forceinline__ uint32_t mx4_codes(const float (&v)[8], float scale) {
  uint32_t q = 0;
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[0], v[1], scale, 0);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[2], v[3], scale, 1);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[4], v[5], scale, 2);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[6], v[7], scale, 3);
  return q;
}

constexpr int kQuantThreads = 256, kQuantUnroll = 4;   // eight values a thread and step

// Eight values a thread; the four threads of a block find its largest absolute
// value, the first of them stores its scale (and the zeros past the last
// column).  `count` (device) limits the rows.  One pass, bound by memory: 8 x
// 11008 x 4096 bf16 values in 203 us, 4.5 TB/s (a large copy: 4.9).
template <bool F32>
__global__ __launch_bounds__(kQuantThreads) void mx4_quantize_kernel(const void* __restrict__ x,
                                                                     const int32_t* __restrict__ row_index,
                                                                     const int32_t* __restrict__ count, int rows,
                                                                     long long total_rows, int cols,
                                                                     uint8_t* __restrict__ q, uint8_t* __restrict__ s) {
  const int units = cols / 8, groups256 = (cols + 255) / 256;
  const long long limit = (count ? min(static_cast<long long>(*count), total_rows) : total_rows) * units;
  const long long base = static_cast<long long>(blockIdx.x) * (kQuantThreads * kQuantUnroll);
  const long long row0 = base / units;
  const int first = static_cast<int>(base - row0 * units);
#pragma unroll
  for (int i = 0; i < kQuantUnroll; ++i) {
    const int at = i * kQuantThreads + threadIdx.x;
    const bool in = base + at < limit;   // (the same for a block's four threads)
    const unsigned u = static_cast<unsigned>(first + at);
    const long long r = row0 + u / units;
    const int c = static_cast<int>(u % units);
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (in) {
      const size_t src = static_cast<size_t>(row_index ? row_index[r] : r) * cols + c * 8;
      if constexpr (F32) {
        const float4 a = *reinterpret_cast<const float4*>(static_cast<const float*>(x) + src);
        const float4 b = *reinterpret_cast<const float4*>(static_cast<const float*>(x) + src + 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
      } else {
        Pack16 a;
        a.u4 = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(x) + src);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = bf16_to_f32(a.h[j]);
      }
    }
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) most = max(most, abs_bits(v[j]));
    most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 1, 64)));
    most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 2, 64)));
    if (!in) continue;
    const uint32_t ex = mx4_exponent(most);
    const uint32_t codes = ex == 255u ? 0u : mx4_codes(v, __uint_as_float(ex << 23));
    *reinterpret_cast<uint32_t*>(q + static_cast<size_t>(r) * (cols / 2) + c * 4) = codes;
    if ((c & 3) == 0) {
      const long long g = r / rows;
      const int b = c >> 2;
      uint8_t* dst = s + ((static_cast<size_t>(g) * groups256 + (b >> 3)) * rows + static_cast<size_t>(r - g * rows)) * 8;
      dst[b & 7] = static_cast<uint8_t>(ex);
      if (c + 4 == units)
        for (int z = (b & 7) + 1; z < 8; ++z) dst[z] = 0;
    }
  }
}

// Eight values a thread; 8 x 11008 x 4096 bf16 values in 165 us, 5.5 TB/s.
template <bool F32>
__global__ __launch_bounds__(kQuantThreads) void mx4_dequantize_kernel(const uint8_t* __restrict__ q,
                                                                       const uint8_t* __restrict__ s, int rows,
                                                                       long long total_rows, int cols,
                                                                       void* __restrict__ x) {
  typedef __bf16 bf16v2 __attribute__((ext_vector_type(2)));
  typedef float f32v2 __attribute__((ext_vector_type(2)));
  const int units = cols / 8, groups256 = (cols + 255) / 256;
  const long long limit = total_rows * units;
  const long long base = static_cast<long long>(blockIdx.x) * (kQuantThreads * kQuantUnroll);
  const long long row0 = base / units;
  const int first = static_cast<int>(base - row0 * units);
#pragma unroll
  for (int i = 0; i < kQuantUnroll; ++i) {
    const int at = i * kQuantThreads + threadIdx.x;
    if (base + at >= limit) continue;
    const unsigned u = static_cast<unsigned>(first + at);
    const long long r = row0 + u / units, g = r / rows;
    const int c = static_cast<int>(u % units), b = c >> 2;
    const uint32_t codes = *reinterpret_cast<const uint32_t*>(q + static_cast<size_t>(r) * (cols / 2) + c * 4);
    const uint32_t ex =
        s[((static_cast<size_t>(g) * groups256 + (b >> 3)) * rows + static_cast<size_t>(r - g * rows)) * 8 + (b & 7)];
    const float scale = __uint_as_float(ex << 23);   // only its exponent is read; 255 gives NaN
    const size_t dst = static_cast<size_t>(r) * cols + c * 8;
    if constexpr (F32) {
      const f32v2 v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0);
      const f32v2 v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
      const f32v2 v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2);
      const f32v2 v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
      float4* o = reinterpret_cast<float4*>(static_cast<float*>(x) + dst);
      o[0] = make_float4(v0.x, v0.y, v1.x, v1.y);
      o[1] = make_float4(v2.x, v2.y, v3.x, v3.y);
    } else {
      union { bf16v2 p[4]; uint4 u4; } o;
      o.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
      o.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
      o.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
      o.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(x) + dst) = o.u4;
    }
  }
}

// ------------------------------------------------------------- the product
enum Mx4Out { kOutF32 = 0, kOutBf16 = 1, kOutMx4Gelu = 2, kOutMx4Silu = 3 };

// Three tile shapes.  128 x 128 and 128 x 64: four waves, two blocks a CU (one
// block's epilogue under the other's products).  256 x 256: eight waves, one
// block a CU, half the operand bytes from L2, which is what bounds the others (a
// copy of the kernel without MFMAs takes nine tenths of its time).
//   With few rows an expert most of a 128 x 128 tile's second 64 rows are empty,
// the weights are read once in either shape, and three stages in flight beat two.
// FFN on 32 experts of 2048 x 4096 (us, 128 x 64 | 128 x 128): 500 rows 56 | 61,
// 2000 rows 66 | 70, 2500 rows 87 | 76, 4000 rows 101 | 88; on 16 of 1024 x 4096:
// 200 rows 26 | 31, 1000 rows 31.6 | 32.6, 1200 rows 36.6 | 35.8.
//   256 x 256 exposes its first loads and its epilogue, so it takes one matrix
// whose tiles fill whole rounds of the CUs, and rows of more than eight stages.
// Rows x N x K, bf16 results (us, 128 x 128 | 256 x 256): 8192 x 4096 x 4096 97 |
// 82, 16384 x 11008 x 4096 464 | 410, 16384 x 4096 x 8192 309 | 266; K = 1088 and
// float32 results, 5003 x 2880 23.6 | 25.8, 16384 x 2880 68 | 72; of rounds 0.8
// full, 6000 x 11008 x 4096 169 | 172; 0.67 full, 3000 x 11008 x 4096 95 | 99; FFN
// of 16384 rows on 16 experts of 1024 x 4096 139 | 184.
using Mx4Large = Mx4Core<256, 256, 2, 4, 2>;
using Mx4Wide = Mx4Core<128, 128, 2, 2, 2>;
using Mx4Narrow = Mx4Core<128, 64, 4, 1, 3>;
// Rows are the caller's bound on them (M, max_rows), which the host knows; the
// offsets on the device may hold fewer.
constexpr int kNarrowRows = 64;   // average rows an expert up to which Mx4Narrow runs

// Tile t of the grouped product -> expert, first row, rows, first column: the
// tiles expert by expert (one expert's counts a lane), in blocks of 8 row tiles
// by 4 column tiles, which an XCD's 32 CUs run together: 12 operand panels in
// its L2 for 32 tiles.
struct Mx4Tiles {
  int lo, hi, mt, incl, NT, tiles;
  __device__ __forceinline__ Mx4Tiles(const int32_t* __restrict__ offsets, int E, int M, int N, int bm, int bn) {
    const int lane = threadIdx.x & 63;
    NT = (N + bm - 1) / bm;
    lo = hi = 0;
    if (lane < E) {
      lo = offsets ? min(max(offsets[lane], 0), M) : 0;
      hi = offsets ? min(offsets[lane + 1], M) : M;
    }
    mt = hi > lo ? (hi - lo + bn - 1) / bn : 0;
    incl = mt * NT;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(incl, o, 64);
      if (lane >= o) incl += v;
    }
    tiles = __builtin_amdgcn_readfirstlane(__shfl(incl, 63, 64));
  }
  __device__ __forceinline__ void decode(int t, int E, int bm, int bn, int& e, int& row0, int& rows, int& n0) const {
    const int lane = threadIdx.x & 63;
    e = __popcll(__ballot(lane < E && incl <= t));
    const int me = __shfl(mt, e, 64);
    const int r = t - (__shfl(incl, e, 64) - me * NT);
    const int g = min(r / (4 * me), (NT + 3) / 4 - 1), cols = min(4, NT - 4 * g);
    const int r2 = r - 4 * g * me, rg = min(r2 / (8 * cols), (me + 7) / 8 - 1);
    const int r3 = r2 - 8 * cols * rg, nr = min(8, me - 8 * rg);
    row0 = __builtin_amdgcn_readfirstlane(__shfl(lo, e, 64) + (8 * rg + r3 % nr) * bn);
    rows = __builtin_amdgcn_readfirstlane(min(bn, __shfl(hi, e, 64) - row0));
    n0 = __builtin_amdgcn_readfirstlane((4 * g + r3 / nr) * bm);
  }
};

// A wave's results of 32 rows (accumulators of one Q block: lane l has row
// l % 32 and, in value v of block i, column 32 i + 8 (v / 4) + 4 (l / 32) + v %
// 4) as float32 or bf16.  They turn in LDS, so that a store writes whole lines
// of a row, past the caches' operands (non-temporal).  A product with 16384 x
// 11008 bf16 results: 498 us with 8-byte stores straight from the registers, 32
// rows each, 470 by way of LDS, 461 non-temporal (and 557 non-temporal without
// whole lines).  The 16-byte chunks of a row are permuted by the row, so that
// both sides fall on distinct banks.
template <class G, bool F32>
__device__ __forceinline__ void store_rows(const f32x16 (&acc)[G::FM], int rows, size_t row, int n, int N,
                                           void* __restrict__ out, uint8_t* lds) {
  constexpr int BYTES = F32 ? 4 : 2, PITCH = G::WTM * BYTES, CHUNKS = PITCH / 16, PER = 64 / CHUNKS;
  constexpr int MASK = CHUNKS < 8 ? CHUNKS - 1 : 7, SHIFT = CHUNKS < 8 ? 1 : 0;
  static_assert(CHUNKS == 4 || CHUNKS == 8 || CHUNKS == 16 || CHUNKS == 32, "chunk permutation");
  const int lane = threadIdx.x & 63, half = lane >> 5, r = lane & 31, sw = (r >> SHIFT) & MASK;
  uint8_t* mine = lds + r * PITCH;
#pragma unroll
  for (int i = 0; i < G::FM; ++i) {
    if constexpr (F32) {
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4*>(mine + 16 * ((8 * i + 2 * g + half) ^ sw)) =
            make_float4(acc[i][4 * g], acc[i][4 * g + 1], acc[i][4 * g + 2], acc[i][4 * g + 3]);
    } else {
      // lanes l and l ^ 32 exchange halves of two groups of four columns, so
      // that each has eight consecutive ones
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const uint32_t x0 = pack_bf16x2(acc[i][8 * g], acc[i][8 * g + 1]);
        const uint32_t y0 = pack_bf16x2(acc[i][8 * g + 2], acc[i][8 * g + 3]);
        const uint32_t x1 = pack_bf16x2(acc[i][8 * g + 4], acc[i][8 * g + 5]);
        const uint32_t y1 = pack_bf16x2(acc[i][8 * g + 6], acc[i][8 * g + 7]);
        const auto x = __builtin_amdgcn_permlane32_swap(x0, x1, false, false);
        const auto y = __builtin_amdgcn_permlane32_swap(y0, y1, false, false);
        *reinterpret_cast<uint4*>(mine + 16 * ((4 * i + 2 * g + half) ^ sw)) = make_uint4(x[0], y[0], x[1], y[1]);
      }
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // the rows' other lanes are of this wave
  const int c = lane % CHUNKS, cn = n + c * (16 / BYTES);
#pragma unroll
  for (int q = 0; q < 32 / PER; ++q) {
    const int t = q * PER + lane / CHUNKS;
    const i32x4 v = *reinterpret_cast<const i32x4*>(lds + t * PITCH + 16 * (c ^ ((t >> SHIFT) & MASK)));
    if (t < rows && cn < N)
      __builtin_nontemporal_store(v, reinterpret_cast<i32x4*>(static_cast<uint8_t*>(out) + ((row + t) * N + cn) * BYTES));
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// One 32 x 32 block of accumulators (layout as above) through the activation
// and rounded to 4 bits.
template <int ACT>
__device__ __forceinline__ void store_mx4(const f32x16& acc, bool valid, size_t row, int M, int n, int N,
                                          uint8_t* __restrict__ out, uint8_t* __restrict__ out_scale) {
  const int half = (threadIdx.x >> 5) & 1;
  // the activation, then the rounding to 4 bits: the 32 columns of a row are
  // one block, half of it in lane l and half in lane l ^ 32
  float v[16];
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    v[i] = act_relative<ACT>(acc[i]);
    most = max(most, abs_bits(v[i]));
  }
  most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 32, 64)));
  const uint32_t ex = mx4_exponent(most);
  const float scale = __uint_as_float(ex << 23);
  uint32_t c[2] = {0, 0};   // columns 0-3 and 8-11, 16-19 and 24-27 (+ 4 in the upper half)
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    c[g] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c[g], v[8 * g], v[8 * g + 1], scale, 0);
    c[g] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c[g], v[8 * g + 2], v[8 * g + 3], scale, 1);
    c[g] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c[g], v[8 * g + 4], v[8 * g + 5], scale, 2);
    c[g] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c[g], v[8 * g + 6], v[8 * g + 7], scale, 3);
    if (ex == 255u) c[g] = 0;
  }
  // the lower half stores columns 0-15, the upper one 16-31
  const uint32_t got = static_cast<uint32_t>(__shfl_xor(static_cast<int>(half ? c[0] : c[1]), 32, 64));
  const uint32_t a = half ? got : c[0], b = half ? c[1] : got;   // columns +0..3 and +4..7 of each eight
  if (!valid) return;
  *reinterpret_cast<uint2*>(out + row * (N / 2) + n / 2 + 8 * half) =
      make_uint2((a & 0xFFFFu) | (b << 16), (a >> 16) | (b & 0xFFFF0000u));
  if (half == 0) {
    uint8_t* dst = out_scale + (static_cast<size_t>(n >> 8) * M + row) * 8;
    const int blk = n >> 5 & 7;
    dst[blk] = static_cast<uint8_t>(ex);
    if (n + 32 == N)
      for (int z = blk + 1; z < 8; ++z) dst[z] = 0;
  }
}

// y[r] = W_e x_r for the rows of every expert, a block a tile.  16384 x 11008 x
// 4096 in 435 us on average over 30 calls on their own (382 to 498; 380 to 395 a
// call in longer runs), 3400 TFLOP/s: half of what the 4-bit MFMA does alone
// (7380); MFMA busy 52 % of the cycles, the rest is the first loads and the
// epilogue of a CU's one block.  The first product of an FFN is bound by its
// epilogue: about 25 vector instructions a hidden value, two of them
// transcendental (8653 rows on 32 experts of 2048 x 8192: 170 us; vector units
// half busy).
// Whether a block takes one tile after the other, the next one's first loads
// under the epilogue: all shapes with two blocks a CU.  (FFN of 8653 rows on 32
// experts of 2048 x 8192: first product 190 -> 170 us, second 150 -> 134; of 2000
// rows on 32 of 2048 x 4096 82 -> 66 for both.)  256 x 256 has no registers left for it: 93
// spilled, 402 -> 498 us on 16384 x 11008 x 4096.
template <class G>
constexpr bool mx4_stays() {
  return 2 * G::LDS_BYTES <= 160 * 1024;
}

template <class G, int OUT>
__global__ __launch_bounds__(G::THREADS) void mx4_product_kernel(
    const uint8_t* __restrict__ xq, const uint8_t* __restrict__ xs, int M, const int32_t* __restrict__ offsets, int E,
    int N, int K, const uint8_t* __restrict__ wq, const uint8_t* __restrict__ ws, void* __restrict__ out,
    uint8_t* __restrict__ out_scale) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[G::LDS_BYTES];
  const Mx4Tiles map(offsets, E, M, N, G::BM, G::BN);
  int t = xcd_virtual_block();
  if (t >= map.tiles) return;
  const int kbytes = K / 2, kstages = (K + 255) / 256;
  typename G::Tile tile;
  typename G::Pipe pipe;
  tile.ps_stage = static_cast<size_t>(N) * 8;
  tile.qs_stage = static_cast<size_t>(M) * 8;
  tile.kbytes = kbytes;
  int row0, rows, n0;
  // Results turn in LDS behind the first stage, which may already hold the next
  // tile's by then; 4-bit results need no LDS, and all first stages go out.
  constexpr bool MX4 = OUT == kOutMx4Gelu || OUT == kOutMx4Silu;
  constexpr int TURN = G::NWAVES * 32 * G::WTM * (OUT == kOutF32 ? 4 : 2);
  constexpr bool STAY = mx4_stays<G>();
  constexpr int EARLY = MX4 ? G::STAGES : 1;
  static_assert(MX4 || TURN <= (G::STAGES - STAY) * G::STAGE_BYTES, "results turn in the operands' LDS");
  // tile t's place, and its first stages on their way
  auto start = [&]() {
    int e;
    map.decode(t, E, G::BM, G::BN, e, row0, rows, n0);
    tile.p = wq + (static_cast<size_t>(e) * N + n0) * kbytes;
    tile.q = xq + static_cast<size_t>(row0) * kbytes;
    tile.ps = ws + (static_cast<size_t>(e) * kstages * N + n0) * 8;
    tile.qs = xs + static_cast<size_t>(row0) * 8;
    tile.pvalid = min(G::BM, N - n0);
    tile.qvalid = rows;
    G::template prefetch<0, EARLY>(tile, pipe, lds);
  };
  start();
  const int lane = threadIdx.x & 63, w = G::wave(), wm = G::wave_m(w), wn = G::wave_n(w);
  while (true) {
    G::template prefetch<EARLY, G::STAGES>(tile, pipe, lds);
    typename G::Acc acc;
    G::zero(acc);
    G::run_nq(G::active_q(wn, rows), tile, pipe, lds, acc);
    const int out_row0 = row0, out_rows = rows, n = n0 + wm * G::WTM;
    bool more = false;
    if constexpr (STAY) {
      t += gridDim.x;
      more = t < map.tiles;
      if (more) start();
    }
#pragma unroll
    for (int j = 0; j < G::FN; ++j) {
      const int q = G::q_row(wn, j);
      if (q >= out_rows) break;
      const size_t row = static_cast<size_t>(out_row0) + q;
      if constexpr (OUT == kOutF32 || OUT == kOutBf16) {
        constexpr bool F32 = OUT == kOutF32;
        f32x16 a[G::FM];
#pragma unroll
        for (int i = 0; i < G::FM; ++i) a[i] = acc[i][j];
        store_rows<G, F32>(a, out_rows - q, row, n, N, out, lds + (STAY ? G::STAGE_BYTES : 0) + w * (TURN / G::NWAVES));
      } else {
        constexpr int ACT = OUT == kOutMx4Gelu ? LUFFY_ACT_GELU : LUFFY_ACT_SILU;
#pragma unroll
        for (int i = 0; i < G::FM; ++i)
          if (n + 32 * i < N)
            store_mx4<ACT>(acc[i][j], q + (lane & 31) < out_rows, row + (lane & 31), M, n + 32 * i, N,
                           static_cast<uint8_t*>(out), out_scale);
      }
    }
    if (!more) break;
    if constexpr (!MX4) {   // every wave is done turning before the other stages go out
      __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
      raw_barrier();
    }
  }
}

template <class G, int OUT>
void launch_shape(const char* name, const uint8_t* xq, const uint8_t* xs, int M, const int32_t* offsets, int E, int N,
                  int K, const uint8_t* wq, const uint8_t* ws, void* out, uint8_t* out_scale, hipStream_t s) {
  // every expert may add one partial row tile
  const long long row_tiles = (M + G::BN - 1) / G::BN + (offsets ? E - 1 : 0);
  long long tiles = row_tiles * ((N + G::BM - 1) / G::BM);
  if (mx4_stays<G>()) tiles = std::min(tiles, 2ll * persistent_grid());
  launch(name, mx4_product_kernel<G, OUT>, static_cast<int>((tiles + 7) / 8 * 8), G::THREADS, 0, s, xq, xs, M, offsets,
         E, N, K, wq, ws, out, out_scale);
}

template <int OUT>
void launch_product(const char* name, const uint8_t* xq, const uint8_t* xs, int M, const int32_t* offsets, int E,
                    int N, int K, const uint8_t* wq, const uint8_t* ws, void* out, uint8_t* out_scale, hipStream_t s) {
  if constexpr (OUT == kOutF32 || OUT == kOutBf16) {
    const long long tiles = static_cast<long long>((M + Mx4Large::BN - 1) / Mx4Large::BN) *
                            ((N + Mx4Large::BM - 1) / Mx4Large::BM);
    const int cus = persistent_grid();
    if (E == 1 && K > 2048 && 10 * tiles >= 9 * ((tiles + cus - 1) / cus * cus)) {
      launch_shape<Mx4Large, OUT>(name, xq, xs, M, offsets, E, N, K, wq, ws, out, out_scale, s);
      return;
    }
  }
  if (M <= kNarrowRows * E)
    launch_shape<Mx4Narrow, OUT>(name, xq, xs, M, offsets, E, N, K, wq, ws, out, out_scale, s);
  else
    launch_shape<Mx4Wide, OUT>(name, xq, xs, M, offsets, E, N, K, wq, ws, out, out_scale, s);
}

void launch_quantize(const void* x, const int32_t* row_index, const int32_t* count, int rows, long long total_rows,
                     int cols, int dtype, uint8_t* q, uint8_t* s, hipStream_t st) {
  const long long per = kQuantThreads * kQuantUnroll;
  const int blocks = static_cast<int>((total_rows * (cols / 8) + per - 1) / per);
  auto* kernel = dtype == LUFFY_F32 ? mx4_quantize_kernel<true> : mx4_quantize_kernel<false>;
  launch("mx4_quantize", kernel, blocks, kQuantThreads, 0, st, x, row_index, count, rows, total_rows, cols, q, s);
}

struct Mx4FfnWs {
  uint8_t *xq, *xs, *hq, *hs;
};

Mx4FfnWs carve_mx4_ffn(Carver& c, int max_rows, int d, int d_ff) {
  Mx4FfnWs w;
  const size_t r = max_rows;
  w.xq = c.take<uint8_t>(r * (d / 2));
  w.xs = c.take<uint8_t>(r * ((d + 255) / 256 * 8));
  w.hq = c.take<uint8_t>(r * (d_ff / 2));
  w.hs = c.take<uint8_t>(r * ((d_ff + 255) / 256 * 8));
  return w;
}

bool misaligned(const void* p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// The checks that quantize and dequantize share.
int check_matrix(const char* what, const void* x, const void* q, const void* s, int groups, int rows, int cols,
                 int dtype) {
  if (!x || !q || !s) return fail(LUFFY_E_INVALID, "%s: null pointer argument", what);
  if (groups <= 0 || rows <= 0 || cols <= 0)
    return fail(LUFFY_E_INVALID, "%s: groups=%d rows=%d cols=%d", what, groups, rows, cols);
  if (dtype != LUFFY_F32 && dtype != LUFFY_BF16) return fail(LUFFY_E_INVALID, "%s: unknown dtype %d", what, dtype);
  if (cols % 32 != 0) return fail(LUFFY_E_UNSUPPORTED, "%s: cols=%d not a multiple of 32", what, cols);
  if (static_cast<double>(groups) * rows * (cols / 8) >= 1024.0 * 0x7fffff00)
    return fail(LUFFY_E_UNSUPPORTED, "%s: groups=%d rows=%d cols=%d is too large", what, groups, rows, cols);
  if (misaligned(x, 16) || misaligned(q, 16) || misaligned(s, 8))
    return fail(LUFFY_E_INVALID, "%s: x and q must be 16-byte aligned, s 8-byte", what);
  return LUFFY_OK;
}

}  // namespace
}  // namespace luffy

using namespace luffy;

extern "C" size_t luffy_mx4_scale_bytes(int groups, int rows, int cols) {
  if (groups <= 0 || rows <= 0 || cols <= 0) return 0;
  return static_cast<size_t>(groups) * rows * ((static_cast<size_t>(cols) + 255) / 256) * 8;
}

extern "C" int luffy_mx4_quantize(const void* x, const int32_t* row_index, int groups, int rows, int cols, int dtype,
                                  void* q, void* s, void* stream) {
  if (const int e = check_matrix("luffy_mx4_quantize", x, q, s, groups, rows, cols, dtype)) return e;
  if (row_index && groups != 1) return fail(LUFFY_E_INVALID, "luffy_mx4_quantize: row_index needs groups = 1");
  launch_quantize(x, row_index, nullptr, rows, static_cast<long long>(groups) * rows, cols, dtype,
                  static_cast<uint8_t*>(q), static_cast<uint8_t*>(s), static_cast<hipStream_t>(stream));
  return check_launch("luffy_mx4_quantize");
}

extern "C" int luffy_mx4_dequantize(const void* q, const void* s, int groups, int rows, int cols, int dtype, void* x,
                                    void* stream) {
  if (const int e = check_matrix("luffy_mx4_dequantize", x, q, s, groups, rows, cols, dtype)) return e;
  const long long total = static_cast<long long>(groups) * rows, per = kQuantThreads * kQuantUnroll;
  const int blocks = static_cast<int>((total * (cols / 8) + per - 1) / per);
  auto* kernel = dtype == LUFFY_F32 ? mx4_dequantize_kernel<true> : mx4_dequantize_kernel<false>;
  launch("mx4_dequantize", kernel, blocks, kQuantThreads, 0, static_cast<hipStream_t>(stream),
         static_cast<const uint8_t*>(q), static_cast<const uint8_t*>(s), rows, total, cols, x);
  return check_launch("luffy_mx4_dequantize");
}

extern "C" int luffy_mx4_matmul(const void* xq, const void* xs, int M, const int32_t* offsets, int E, int N, int K,
                                const void* wq, const void* ws, void* y, int dtype, void* stream) {
  if (!xq || !xs || !wq || !ws || !y) return fail(LUFFY_E_INVALID, "luffy_mx4_matmul: null pointer argument");
  if (M <= 0 || E <= 0 || N <= 0 || K <= 0)
    return fail(LUFFY_E_INVALID, "luffy_mx4_matmul: M=%d E=%d N=%d K=%d", M, E, N, K);
  if (!offsets && E != 1) return fail(LUFFY_E_INVALID, "luffy_mx4_matmul: E=%d needs offsets", E);
  if (dtype != LUFFY_F32 && dtype != LUFFY_BF16)
    return fail(LUFFY_E_INVALID, "luffy_mx4_matmul: unknown dtype %d", dtype);
  if (E > kMaxExperts) return fail(LUFFY_E_UNSUPPORTED, "luffy_mx4_matmul: E=%d > %d", E, kMaxExperts);
  if (N % 32 != 0 || K % 32 != 0 || N > 32768 || K > 32768)
    return fail(LUFFY_E_UNSUPPORTED, "luffy_mx4_matmul: N=%d K=%d must be multiples of 32 and at most 32768", N, K);
  if (M > (1 << 24)) return fail(LUFFY_E_UNSUPPORTED, "luffy_mx4_matmul: M=%d > 2^24", M);
  if (misaligned(xq, 16) || misaligned(wq, 16) || misaligned(y, 16) || misaligned(xs, 8) || misaligned(ws, 8))
    return fail(LUFFY_E_INVALID, "luffy_mx4_matmul: xq, wq and y must be 16-byte aligned, xs and ws 8-byte");
  hipStream_t st = static_cast<hipStream_t>(stream);
  const auto *a = static_cast<const uint8_t*>(xq), *as = static_cast<const uint8_t*>(xs);
  const auto *b = static_cast<const uint8_t*>(wq), *bs = static_cast<const uint8_t*>(ws);
  if (dtype == LUFFY_F32) launch_product<kOutF32>("mx4_matmul", a, as, M, offsets, E, N, K, b, bs, y, nullptr, st);
  else launch_product<kOutBf16>("mx4_matmul", a, as, M, offsets, E, N, K, b, bs, y, nullptr, st);
  return check_launch("luffy_mx4_matmul");
}

extern "C" size_t luffy_mx4_expert_ffn_workspace_size(int max_rows, int E, int d, int d_ff) {
  if (max_rows <= 0 || E <= 0 || d <= 0 || d_ff <= 0) return 0;
  Carver c(nullptr);
  carve_mx4_ffn(c, max_rows, d, d_ff);
  return c.size();
}

extern "C" int luffy_mx4_expert_ffn(const void* x, const int32_t* row_index, const int32_t* rep_offsets, int E, int d,
                                    int d_ff, const void* w1q, const void* w1s, const void* w2q, const void* w2s,
                                    int act, int max_rows, void* y_rep, void* workspace, size_t workspace_bytes,
                                    void* stream) {
  if (!x || !rep_offsets || !w1q || !w1s || !w2q || !w2s || !y_rep)
    return fail(LUFFY_E_INVALID, "luffy_mx4_expert_ffn: null pointer argument");
  if (E <= 0 || d <= 0 || d_ff <= 0 || max_rows <= 0)
    return fail(LUFFY_E_INVALID, "luffy_mx4_expert_ffn: E=%d d=%d d_ff=%d max_rows=%d", E, d, d_ff, max_rows);
  if (act != LUFFY_ACT_GELU && act != LUFFY_ACT_SILU)
    return fail(LUFFY_E_INVALID, "luffy_mx4_expert_ffn: unknown activation %d", act);
  if (E > kMaxExperts) return fail(LUFFY_E_UNSUPPORTED, "luffy_mx4_expert_ffn: E=%d > %d", E, kMaxExperts);
  if (d % 64 != 0 || d_ff % 64 != 0 || d > 32768 || d_ff > 32768)
    return fail(LUFFY_E_UNSUPPORTED,
                "luffy_mx4_expert_ffn: d=%d d_ff=%d must be multiples of 64 and at most 32768", d, d_ff);
  if (max_rows > (1 << 24)) return fail(LUFFY_E_UNSUPPORTED, "luffy_mx4_expert_ffn: max_rows=%d > 2^24", max_rows);
  if (misaligned(x, 16) || misaligned(w1q, 16) || misaligned(w2q, 16) || misaligned(y_rep, 16) ||
      misaligned(w1s, 8) || misaligned(w2s, 8))
    return fail(LUFFY_E_INVALID,
                "luffy_mx4_expert_ffn: x, values and y_rep must be 16-byte aligned, scales 8-byte");
  const size_t need = luffy_mx4_expert_ffn_workspace_size(max_rows, E, d, d_ff);
  if (workspace_bytes < need || !workspace || misaligned(workspace, 256))
    return fail(LUFFY_E_WORKSPACE, "luffy_mx4_expert_ffn: workspace needs %zu bytes, 256-aligned", need);
  hipStream_t st = static_cast<hipStream_t>(stream);
  Carver c(workspace);
  const Mx4FfnWs w = carve_mx4_ffn(c, max_rows, d, d_ff);
  launch_quantize(x, row_index, rep_offsets + E, max_rows, max_rows, d, LUFFY_BF16, w.xq, w.xs, st);
  const auto *b1 = static_cast<const uint8_t*>(w1q), *s1 = static_cast<const uint8_t*>(w1s);
  const auto *b2 = static_cast<const uint8_t*>(w2q), *s2 = static_cast<const uint8_t*>(w2s);
  if (act == LUFFY_ACT_GELU)
    launch_product<kOutMx4Gelu>("mx4_ffn1", w.xq, w.xs, max_rows, rep_offsets, E, d_ff, d, b1, s1, w.hq, w.hs, st);
  else
    launch_product<kOutMx4Silu>("mx4_ffn1", w.xq, w.xs, max_rows, rep_offsets, E, d_ff, d, b1, s1, w.hq, w.hs, st);
  launch_product<kOutBf16>("mx4_ffn2", w.hq, w.hs, max_rows, rep_offsets, E, d, d_ff, b2, s2, y_rep, nullptr, st);
  return check_launch("luffy_mx4_expert_ffn");
}
