// luffy_mx8_quantize and luffy_mx8_dequantize: matrices of microscaled 8-bit
// integers, in which activations are kept for the backward.
#include <algorithm>

#include "luffy_common.h"
#include "mx8.h"

namespace luffy {
namespace {

// Eight values a thread and step; two steps, for float32 results one (us, with one, two
// and four steps: 65536 x 2048 bf16 to 8 bits 83, 85, 92, back 71, 66, 67; 16384 x 4096
// float32 to 8 bits 80, 82, 83, back 58, 79, 84; 3001 x 1088 float32 7.3, 7.3, 8.7 and
// 8.3, 7.6, 8.0).
constexpr int kThreads = 256, kQuantizeSteps = 2;
constexpr int dequantize_steps(bool f32) { return f32 ? 1 : 2; }

// Eight values a thread; a block's four threads find its largest absolute value,
// the first of them stores the scale (and the zeros past the last column).  Bound by
// HBM: 65536 x 2048 bf16 85 us, 4.8 TB/s; back to bf16 66 us, 6.2 TB/s (the values are
// still in the last-level cache in part).  Loads and stores are whole lines.
template <bool F32>
__global__ __launch_bounds__(kThreads) void mx8_quantize_kernel(const void* __restrict__ x, int rows, int cols,
                                                                uint8_t* __restrict__ q, uint8_t* __restrict__ s) {
  const int units = cols / 8;
  const long long limit = static_cast<long long>(rows) * units;
  const long long base = static_cast<long long>(blockIdx.x) * (kThreads * kQuantizeSteps);
  const long long row0 = base / units;
  const int first = static_cast<int>(base - row0 * units);
#pragma unroll
  for (int i = 0; i < kQuantizeSteps; ++i) {
    const int at = i * kThreads + threadIdx.x;
    const bool in = base + at < limit;   // (the same for a block's four threads)
    const unsigned u = static_cast<unsigned>(first + at);
    const long long r = row0 + u / units;
    const int c = static_cast<int>(u % units);
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (in) {
      const size_t src = static_cast<size_t>(r) * cols + c * 8;
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
    for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(v[j]) & 0x7FFFFFFFu);
    most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 1, 64)));
    most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 2, 64)));
    if (!in) continue;
    const uint32_t ex = mx8_exponent(most);
    const float inv = mx8_inverse(min(ex, 248u));
    uint2 w = make_uint2(mx8_pack(v[0], v[1], v[2], v[3], inv), mx8_pack(v[4], v[5], v[6], v[7], inv));
    if (ex == 255u) w = make_uint2(0, 0);
    *reinterpret_cast<uint2*>(q + static_cast<size_t>(r) * cols + c * 8) = w;
    if ((c & 3) == 0) {
      const int b = c >> 2;
      uint8_t* dst = s + (static_cast<size_t>(b >> 3) * rows + static_cast<size_t>(r)) * 8;
      dst[b & 7] = static_cast<uint8_t>(ex);
      if (c + 4 == units)
        for (int z = (b & 7) + 1; z < 8; ++z) dst[z] = 0;
    }
  }
}

template <bool F32>
__global__ __launch_bounds__(kThreads) void mx8_dequantize_kernel(const uint8_t* __restrict__ q,
                                                                  const uint8_t* __restrict__ s, int rows, int cols,
                                                                  void* __restrict__ x) {
  constexpr int kSteps = dequantize_steps(F32);
  const int units = cols / 8;
  const long long limit = static_cast<long long>(rows) * units;
  const long long base = static_cast<long long>(blockIdx.x) * (kThreads * kSteps);
  const long long row0 = base / units;
  const int first = static_cast<int>(base - row0 * units);
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int at = i * kThreads + threadIdx.x;
    if (base + at >= limit) continue;
    const unsigned u = static_cast<unsigned>(first + at);
    const long long r = row0 + u / units;
    const int c = static_cast<int>(u % units), b = c >> 2;
    const size_t to = static_cast<size_t>(r) * cols + c * 8;
    const uint2 w = *reinterpret_cast<const uint2*>(q + to);
    const float f = mx8_scale(s[(static_cast<size_t>(b >> 3) * rows + static_cast<size_t>(r)) * 8 + (b & 7)]);
    float lo[4], hi[4];
    mx8_unpack(w.x, f, lo);
    mx8_unpack(w.y, f, hi);
    if constexpr (F32) {
      float4* o = reinterpret_cast<float4*>(static_cast<float*>(x) + to);
      o[0] = make_float4(lo[0], lo[1], lo[2], lo[3]);
      o[1] = make_float4(hi[0], hi[1], hi[2], hi[3]);
    } else {
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(x) + to) =
          make_uint4(pack_bf16x2(lo[0], lo[1]), pack_bf16x2(lo[2], lo[3]), pack_bf16x2(hi[0], hi[1]),
                     pack_bf16x2(hi[2], hi[3]));
    }
  }
}

long long mx8_blocks(int rows, int cols, int steps) {
  const long long per = kThreads * steps;
  return (static_cast<long long>(rows) * (cols / 8) + per - 1) / per;
}
constexpr long long kMaxValues = 1ll << 34;   // (a grid has fewer than 2^32 threads)

int mx8_check(const char* fn, const void* x, const void* q, const void* s, int rows, int cols, int dtype) {
  if (!x || !q || !s) return fail(LUFFY_E_INVALID, "%s: null pointer argument", fn);
  if (rows <= 0 || cols <= 0) return fail(LUFFY_E_INVALID, "%s: rows=%d cols=%d must be positive", fn, rows, cols);
  if (dtype != LUFFY_F32 && dtype != LUFFY_BF16) return fail(LUFFY_E_INVALID, "%s: unknown dtype %d", fn, dtype);
  if (cols % 32 != 0) return fail(LUFFY_E_UNSUPPORTED, "%s: cols=%d not a multiple of 32", fn, cols);
  if (cols > 32768) return fail(LUFFY_E_UNSUPPORTED, "%s: cols=%d > 32768", fn, cols);
  if (static_cast<long long>(rows) * cols > kMaxValues)
    return fail(LUFFY_E_UNSUPPORTED, "%s: %d x %d is more than 2^34 values", fn, rows, cols);
  const uintptr_t bits = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(q);
  if ((bits & 15u) || (reinterpret_cast<uintptr_t>(s) & 7u))
    return fail(LUFFY_E_INVALID, "%s: x and q must be 16-byte, s 8-byte aligned", fn);
  return LUFFY_OK;
}

}  // namespace
}  // namespace luffy

using namespace luffy;

extern "C" int luffy_mx8_quantize(const void* x, int rows, int cols, int dtype, void* q, void* s, void* stream) {
  const int st = mx8_check("luffy_mx8_quantize", x, q, s, rows, cols, dtype);
  if (st != LUFFY_OK) return st;
  const bool f32 = dtype == LUFFY_F32;
  launch("mx8_quantize", f32 ? mx8_quantize_kernel<true> : mx8_quantize_kernel<false>,
         static_cast<int>(mx8_blocks(rows, cols, kQuantizeSteps)), kThreads, 0, static_cast<hipStream_t>(stream), x,
         rows, cols, static_cast<uint8_t*>(q), static_cast<uint8_t*>(s));
  return check_launch("luffy_mx8_quantize");
}

extern "C" int luffy_mx8_dequantize(const void* q, const void* s, int rows, int cols, int dtype, void* x,
                                    void* stream) {
  const int st = mx8_check("luffy_mx8_dequantize", x, q, s, rows, cols, dtype);
  if (st != LUFFY_OK) return st;
  const bool f32 = dtype == LUFFY_F32;
  launch("mx8_dequantize", f32 ? mx8_dequantize_kernel<true> : mx8_dequantize_kernel<false>,
         static_cast<int>(mx8_blocks(rows, cols, dequantize_steps(f32))), kThreads, 0,
         static_cast<hipStream_t>(stream), static_cast<const uint8_t*>(q), static_cast<const uint8_t*>(s), rows, cols, x);
  return check_launch("luffy_mx8_dequantize");
}
