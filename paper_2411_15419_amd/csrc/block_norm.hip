// luffy_block_norm and luffy_block_norm_backward: the residual stream around a
// layer.
//   N(a; w, b) = (a - m) r w + b,  r = 1 / sqrt(mean((a - m)^2) + eps),
//   m = mean(a) (layer) or 0 (rms)
//   o = res_scale x + g N(y; w_post, b_post),  u = N(o; w_pre, b_pre)
// Every row is read once and kept in registers between its statistics and its
// results, so both directions are bound by HBM.  A row belongs to a team: part
// of a wave, a wave, or the waves of a block; lane `sub` of a team of LT lanes
// has the 8-value chunks sub, sub + LT, ... of its row.  Means are taken before
// deviations (no difference of large sums), all in float32.
#include <algorithm>
#include <initializer_list>

#include "luffy_common.h"

namespace luffy {
namespace {

// Eight consecutive values of a row as they are stored.
template <bool BF16>
struct Chunk {
  uint4 u[BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const void* base, size_t at) {
    if constexpr (BF16) {
      u[0] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + at);
    } else {
      const uint4* p = reinterpret_cast<const uint4*>(static_cast<const float*>(base) + at);
      u[0] = p[0];
      u[1] = p[1];
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < (BF16 ? 1 : 2); ++i) u[i] = make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    if constexpr (BF16) {
      const uint32_t w[4] = {u[0].x, u[0].y, u[0].z, u[0].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    } else {
      const uint32_t w[8] = {u[0].x, u[0].y, u[0].z, u[0].w, u[1].x, u[1].y, u[1].z, u[1].w};
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
    }
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
    if constexpr (BF16) {
      u[0] = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]),
                        pack_bf16x2(f[6], f[7]));
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        u[i] = make_uint4(__float_as_uint(f[4 * i]), __float_as_uint(f[4 * i + 1]), __float_as_uint(f[4 * i + 2]),
                          __float_as_uint(f[4 * i + 3]));
    }
  }
  __device__ __forceinline__ void store(void* base, size_t at) const {
    if constexpr (BF16) {
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + at) = u[0];
    } else {
      uint4* p = reinterpret_cast<uint4*>(static_cast<float*>(base) + at);
      p[0] = u[0];
      p[1] = u[1];
    }
  }
};

__device__ __forceinline__ void load8(const float* p, float (&f)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void store8(float* p, const float (&f)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}

// Sums over a team's lanes; every lane ends with the same sums.  WAVES = 1: the
// team is lt <= 64 consecutive lanes (a power of two).  WAVES > 1: by way of LDS, all
// teams of the block together; `turn` takes the rounds of a row through three
// buffers, so that a buffer is written again only after a barrier that follows its
// reads.
template <int DPP, int ROWS = 0xF>
__device__ __forceinline__ float dpp_f32(float x) {
  return __uint_as_float(static_cast<uint32_t>(
      __builtin_amdgcn_update_dpp(0, static_cast<int>(__float_as_uint(x)), DPP, ROWS, 0xF, false)));
}
template <int WAVES, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], int lt, float (*lds)[16][4], int& turn) {
  // inside rows of 16 lanes
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] += dpp_f32<0xB1>(v[i]);    // quad_perm [1, 0, 3, 2]
    v[i] += dpp_f32<0x4E>(v[i]);    // quad_perm [2, 3, 0, 1]
    v[i] += dpp_f32<0x141>(v[i]);   // row_half_mirror
    if (WAVES > 1 || lt > 8) v[i] += dpp_f32<0x140>(v[i]);   // row_mirror
  }
  if (WAVES == 1 && lt <= 16) return;
  if (WAVES == 1 && lt == 32) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], 16, 64);
    return;
  }
  // the rows' sums to the last lane
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] += dpp_f32<0x142, 0xA>(v[i]);   // row_bcast:15 to rows 1 and 3
    v[i] += dpp_f32<0x143, 0xC>(v[i]);   // row_bcast:31 to rows 2 and 3
  }
  if constexpr (WAVES == 1) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      v[i] = __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(__float_as_uint(v[i])), 63)));
  } else {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, first = w / WAVES * WAVES;
    if (lane == 63) {
#pragma unroll
      for (int i = 0; i < N; ++i) lds[turn][w][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < WAVES; ++j) s += lds[turn][first + j][i];
      v[i] = s;
    }
    turn = turn == 2 ? 0 : turn + 1;
  }
}

struct NormArgs {
  const void *x, *y;
  const float *w_post, *b_post, *w_pre, *b_pre;
  const void* gate;
  int gate_kind;
  int T, d, layer;
  float eps, res_scale;
  void *o, *u;
};

// Mean (layer) and 1 / sqrt(variance + eps) of the row held in c.
template <bool BF16, int CH, int WAVES>
__device__ __forceinline__ void row_stats(const Chunk<BF16> (&c)[CH], int chunks, int sub, int lt, float inv_d,
                                          bool layer, float eps, float (*lds)[16][4], int& turn, float& mean,
                                          float& r) {
  mean = 0.f;
  if (layer) {
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      float f[8];
      c[i].get(f);   // zeros past the row
#pragma unroll
      for (int j = 0; j < 8; ++j) s[0] += f[j];
    }
    team_sum<WAVES>(s, lt, lds, turn);
    mean = s[0] * inv_d;
  }
  float q[1] = {0.f};
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    if (sub + i * lt >= chunks) break;
    float f[8];
    c[i].get(f);
#pragma unroll
    for (int j = 0; j < 8; ++j) q[0] = fmaf(f[j] - mean, f[j] - mean, q[0]);
  }
  team_sum<WAVES>(q, lt, lds, turn);
  r = 1.0f / sqrtf(fmaf(q[0], inv_d, eps));
}

// A row a team, in registers from its loads to its stores.  Bounded by HBM: 8192 x
// 1024 bf16, layer norms and a token gate, 16.7 us, 5.0 TB/s; 16384 x 4096 129 us, 5.2
// TB/s (a large copy: 4.9).  One row of 4096: 2.7 us, a launch and its loads' latency.
// (float32 rows past 16384 columns: 32 registers spill; 2048 x 32768 364 us, 3.7 TB/s.)
template <bool BF16, int CH, int WAVES>
__global__ __launch_bounds__(WAVES > 1 ? WAVES * 64 : 256) void block_norm_kernel(NormArgs a, int lt_log2) {
  __shared__ float lds[3][16][4];
  int turn = 0;
  const int lt = WAVES > 1 ? WAVES * 64 : 1 << lt_log2;
  const int teams = WAVES > 1 ? 1 : 256 >> lt_log2;   // a block's
  const int sub = WAVES > 1 ? threadIdx.x : threadIdx.x & (lt - 1);
  const int chunks = a.d >> 3;
  const float inv_d = 1.0f / static_cast<float>(a.d);
  for (long long t0 = static_cast<long long>(blockIdx.x) * teams; t0 < a.T;
       t0 += static_cast<long long>(gridDim.x) * teams) {
    const long long tt = t0 + (WAVES > 1 ? 0 : threadIdx.x >> lt_log2);
    if (tt >= a.T) break;   // a whole team: its sums are its own
    const size_t row = static_cast<size_t>(tt) * a.d;
    Chunk<BF16> x[CH], y[CH], g[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = sub + i * lt;
      x[i].zero();
      y[i].zero();
      g[i].zero();
      if (c < chunks) {
        x[i].load(a.x, row + 8 * c);
        if (a.y) {
          y[i].load(a.y, row + 8 * c);
          if (a.gate_kind == LUFFY_GATE_TOKEN) g[i].load(a.gate, row + 8 * c);
        }
      }
    }
    if (a.y) {
      float mean = 0.f, r = 1.f;
      if (a.w_post) row_stats<BF16, CH, WAVES>(y, chunks, sub, lt, inv_d, a.layer, a.eps, lds, turn, mean, r);
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int c = sub + i * lt;
        if (c >= chunks) break;
        float v[8], xf[8];
        y[i].get(v);
        x[i].get(xf);
        if (a.w_post) {
          float w[8], b[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
          load8(a.w_post + 8 * c, w);
          if (a.b_post) load8(a.b_post + 8 * c, b);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = fmaf((v[j] - mean) * r, w[j], b[j]);
        }
        if (a.gate_kind != LUFFY_GATE_NONE) {
          float gf[8];
          if (a.gate_kind == LUFFY_GATE_TOKEN) g[i].get(gf);
          else load8(static_cast<const float*>(a.gate) + 8 * c, gf);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] *= gf[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaf(a.res_scale, xf[j], v[j]);
        x[i].set(v);   // the stream as it is stored: what u norms
        x[i].store(a.o, row + 8 * c);
      }
    }
    if (a.u) {
      float mean, r;
      row_stats<BF16, CH, WAVES>(x, chunks, sub, lt, inv_d, a.layer, a.eps, lds, turn, mean, r);
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int c = sub + i * lt;
        if (c >= chunks) break;
        float v[8], w[8], b[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        x[i].get(v);
        load8(a.w_pre + 8 * c, w);
        if (a.b_pre) load8(a.b_pre + 8 * c, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaf((v[j] - mean) * r, w[j], b[j]);
        x[i].set(v);
        x[i].store(a.u, row + 8 * c);
      }
    }
  }
}

// ---------------------------------------------------------------- backward
// Of one row, with ohat = (o - m_o) r_o and yhat = (y - m_y) r_y:
//   q = du w_pre,  dO = do + r_o (q - [mean q] - ohat mean(q ohat))
//   dx = res_scale dO,  dv = g dO,  dg = dO v
//   p = dv w_post,  dy = r_y (p - [mean p] - yhat mean(p yhat))
// ([] for layer norms only), and over the rows dw_pre = sum du ohat, db_pre =
// sum du, dw_post = sum dv yhat, db_post = sum dv and a channel gate's dg.  The
// row sums come in two rounds (rms) or three: means; squares and q (o - m_o);
// p (y - m_y).
// The sums over rows: a thread keeps the same columns for every row it takes
// and adds them up in registers, a block's teams are added in LDS, and the
// blocks' sums go through the workspace to block_norm_reduce_kernel, all in a
// fixed order.
//   Eight to twelve waves a block, one block a CU (its registers, and few sums to add up
// at the end); bf16 rows are fetched while the rows before them are worked on, and a lane
// holds its columns' weights.  16384 x 4096 bf16: 200 us and 7 us for the sums, 3.9
// TB/s in all (a large copy: 4.9); 272 and 25 us with two blocks a CU, nothing in
// flight and row sums by ds_bpermute.  3001 x 1088 float32 31 and 6 us: four rows a
// team, bound by their chains of loads and row sums.
//   Two kinds of rows have more sums a lane than registers.  Past 8192 columns 16 waves
// have 128 a lane for up to 160 sums: 121 to 683 spill, and bytes that take 164 us take
// 479 (4096 x 16384 bf16, rms; 204 as 8192 x 8192), 714 with biases and layer norms, as
// float32 1070 and 1405 for 329.  bf16 rows on three, five and six waves with bias
// gradients, on blocks of nine to twelve waves, spill 20 to 28 (8192 x 2880 with biases and
// layer norms 99 us, without 75).
constexpr int kSums = 5;   // w_pre, b_pre, w_post, b_post, gate

struct NormBwdArgs {
  const void *y, *o, *dout, *du;
  const float *w_post, *b_post, *w_pre;
  const void* gate;
  int gate_kind;
  int T, d, layer;
  float eps, res_scale;
  void *dx, *dy, *dgate;
  float* sum[kSums];   // results; a null one is not wanted
};

// Threads of a block: as many whole teams as about eight waves hold, twelve where
// fewer would be one team.
constexpr int bwd_threads(int waves) {
  return 64 * (waves == 16 ? 16 : waves == 3 ? 9 : waves == 5 ? 10 : waves == 6 ? 12 : waves == 7 ? 7 : 8);
}

// BIAS: db_pre or db_post is wanted.
template <bool BF16, int CH, int WAVES, bool BIAS>
__global__ __launch_bounds__(bwd_threads(WAVES)) void block_norm_backward_kernel(NormBwdArgs a, int lt_log2,
                                                                                 float* __restrict__ part) {
  constexpr int kThreads = bwd_threads(WAVES);
  constexpr bool AHEAD = BF16 && WAVES < 16;
  __shared__ float lds[3][16][4];
  int turn = 0;
  const int lt = WAVES > 1 ? WAVES * 64 : 1 << lt_log2;
  const int teams = WAVES > 1 ? kThreads / (WAVES * 64) : kThreads >> lt_log2;
  const int team = WAVES > 1 ? threadIdx.x / (WAVES * 64) : threadIdx.x >> lt_log2;
  const int sub = WAVES > 1 ? threadIdx.x % (WAVES * 64) : threadIdx.x & (lt - 1);
  const int chunks = a.d >> 3;
  const float inv_d = 1.0f / static_cast<float>(a.d);
  float acc[kSums][CH][8];   // (without BIAS two of them are not touched)
#pragma unroll
  for (int p = 0; p < kSums; ++p)
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[p][i][j] = 0.f;
  struct Rows {
    Chunk<BF16> y[CH], o[CH], g[CH], dn[CH], du[CH];
  };
  // (a team past the last row has zeros, and stores nothing)
  auto load = [&](long long tt, Rows& r) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = sub + i * lt;
      r.y[i].zero();
      r.o[i].zero();
      r.g[i].zero();
      r.dn[i].zero();
      r.du[i].zero();
      if (tt < a.T && c < chunks) {
        const size_t at = static_cast<size_t>(tt) * a.d + 8 * c;
        if (a.y) r.y[i].load(a.y, at);
        if (a.dout) r.dn[i].load(a.dout, at);
        if (a.du) {
          r.o[i].load(a.o, at);
          r.du[i].load(a.du, at);
        }
        if (a.gate_kind == LUFFY_GATE_TOKEN) r.g[i].load(a.gate, at);
      }
    }
  };
  // a lane's columns are the same in every row: their weights stay in registers
  // where there is one chunk of them
  constexpr bool HOLD = CH == 1 && WAVES < 16;
  float held[3][8];   // w_pre, w_post, a channel gate
  if constexpr (HOLD) {
    const int c = 8 * min(sub, chunks - 1);
    if (a.du) load8(a.w_pre + c, held[0]);
    if (a.w_post) load8(a.w_post + c, held[1]);
    if (a.gate_kind == LUFFY_GATE_CHANNEL) load8(static_cast<const float*>(a.gate) + c, held[2]);
  }
  auto weights = [&](int which, const float* from, int c, float (&w)[8]) {
    if constexpr (HOLD) {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = held[which][j];
    } else {
      load8(from + 8 * c, w);
    }
  };
  const long long step = static_cast<long long>(gridDim.x) * teams;
  long long t0 = static_cast<long long>(blockIdx.x) * teams;
  Rows cur, ahead;
  if constexpr (AHEAD) load(t0 + team, ahead);
  for (; t0 < a.T; t0 += step) {
    const long long tt = t0 + team;
    if constexpr (AHEAD) {
      cur = ahead;
      load(tt + step, ahead);
    } else {
      load(tt, cur);
    }
    const bool valid = tt < a.T;
    if (WAVES == 1 && !valid) break;   // a whole team: its sums are its own
    const size_t row = static_cast<size_t>(valid ? tt : 0) * a.d;
    const auto& y = cur.y;
    const auto& o = cur.o;
    const auto& g = cur.g;
    const auto& dn = cur.dn;
    const auto& du = cur.du;
    float mo = 0.f, my = 0.f;
    if (a.layer) {
      float s[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        float f[8], h[8];
        o[i].get(f);
        y[i].get(h);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          s[0] += f[j];
          s[1] += h[j];
        }
      }
      team_sum<WAVES>(s, lt, lds, turn);
      mo = s[0] * inv_d;
      my = s[1] * inv_d;
    }
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = sub + i * lt;
      if (c >= chunks) break;
      if (a.du) {
        float f[8], q[8], w[8];
        o[i].get(f);
        du[i].get(q);
        weights(0, a.w_pre, c, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float dev = f[j] - mo;
          s[0] = fmaf(dev, dev, s[0]);
          s[1] = fmaf(q[j] * w[j], dev, s[1]);
          s[2] = fmaf(q[j], w[j], s[2]);
        }
      }
      if (a.w_post) {
        float f[8];
        y[i].get(f);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[3] = fmaf(f[j] - my, f[j] - my, s[3]);
      }
    }
    if (a.du || a.w_post) team_sum<WAVES>(s, lt, lds, turn);
    const float ro = 1.0f / sqrtf(fmaf(s[0], inv_d, a.eps)), ry = 1.0f / sqrtf(fmaf(s[3], inv_d, a.eps));
    const float qo = s[1] * ro * inv_d, qm = a.layer ? s[2] * inv_d : 0.f;   // mean(q ohat), mean q
    float ps[2] = {0.f, 0.f};
    Chunk<false> p[CH];   // p, kept in float32 for dy
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = sub + i * lt;
      if (c >= chunks) break;
      float dt[8];
      dn[i].get(dt);
      if (a.du) {
        float f[8], q[8], w[8];
        o[i].get(f);
        du[i].get(q);
        weights(0, a.w_pre, c, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float oh = (f[j] - mo) * ro;
          if (valid) acc[0][i][j] = fmaf(q[j], oh, acc[0][i][j]);
          if (BIAS) acc[1][i][j] += q[j];
          dt[j] += ro * (fmaf(q[j], w[j], -qm) - oh * qo);
        }
      }
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = a.res_scale * dt[j];
      Chunk<BF16> st;
      st.set(v);
      if (valid) st.store(a.dx, row + 8 * c);
      if (!a.y) continue;
      float yh[8];
      y[i].get(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) yh[j] = (v[j] - my) * ry;
      float w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
      if (a.w_post) {
        float b[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        weights(1, a.w_post, c, w);
        if (a.b_post) load8(a.b_post + 8 * c, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaf(yh[j], w[j], b[j]);
      }
      if (a.gate_kind != LUFFY_GATE_NONE) {
        float gf[8], dg[8];
        if (a.gate_kind == LUFFY_GATE_TOKEN) g[i].get(gf);
        else weights(2, static_cast<const float*>(a.gate), c, gf);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          dg[j] = dt[j] * v[j];
          dt[j] *= gf[j];
        }
        if (a.gate_kind == LUFFY_GATE_TOKEN) {
          st.set(dg);
          if (valid && a.dgate) st.store(a.dgate, row + 8 * c);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (valid) acc[4][i][j] += dg[j];
        }
      }
      if (a.w_post) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (valid) acc[2][i][j] = fmaf(dt[j], yh[j], acc[2][i][j]);
          if (BIAS && valid) acc[3][i][j] += dt[j];
          dt[j] *= w[j];
          ps[0] = fmaf(dt[j], yh[j], ps[0]);
          ps[1] += dt[j];
        }
      }
      p[i].set(dt);
    }
    if (!a.y) continue;
    if (a.w_post) team_sum<WAVES>(ps, lt, lds, turn);
    const float py = ps[0] * inv_d, pm = a.layer ? ps[1] * inv_d : 0.f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = sub + i * lt;
      if (c >= chunks) break;
      float v[8], pf[8];
      p[i].get(pf);
      if (a.w_post) {
        y[i].get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) pf[j] = ry * (pf[j] - pm - (v[j] - my) * ry * py);
      }
      Chunk<BF16> st;
      st.set(pf);
      if (valid) st.store(a.dy, row + 8 * c);
    }
  }
  // sums over rows: the block's teams in LDS, one sum of kSums at a time
  __shared__ __attribute__((aligned(16))) float cols[kThreads == WAVES * 64 ? 1 : kThreads * 8 * CH];
#pragma unroll
  for (int p = 0; p < kSums; ++p) {
    if (!a.sum[p]) continue;
    float* dst = gridDim.x > 1 ? part + (static_cast<size_t>(blockIdx.x) * kSums + p) * a.d : a.sum[p];
    if constexpr (kThreads == WAVES * 64) {
#pragma unroll
      for (int i = 0; i < CH; ++i)
        if (sub + i * lt < chunks) store8(dst + 8 * (sub + i * lt), acc[p][i]);
    } else {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < CH; ++i) store8(cols + (static_cast<size_t>(team) * CH * lt + i * lt + sub) * 8, acc[p][i]);
      __syncthreads();
      for (int c = threadIdx.x; c < a.d; c += kThreads) {
        float s = 0.f;
        for (int m = 0; m < teams; ++m) s += cols[static_cast<size_t>(m) * CH * lt * 8 + c];
        dst[c] = s;
      }
    }
  }
}

// Sums of the blocks' parts: 64 columns of one sum a block, a wave a sixteenth of
// the parts (its loads are in flight together).
__global__ __launch_bounds__(1024) void block_norm_reduce_kernel(const float* __restrict__ part, int blocks, int d,
                                                                 NormBwdArgs a) {
  __shared__ float lds[16][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int p = blockIdx.y, c = blockIdx.x * 64 + lane;   // d is a multiple of 64
  float* out = p == 0 ? a.sum[0] : p == 1 ? a.sum[1] : p == 2 ? a.sum[2] : p == 3 ? a.sum[3] : a.sum[4];
  if (!out) return;
  float s = 0.f;
#pragma unroll 16
  for (int b = w; b < blocks; b += 16) s += part[(static_cast<size_t>(b) * kSums + p) * d + c];
  lds[w][lane] = s;
  __syncthreads();
  if (w == 0) {
#pragma unroll
    for (int j = 1; j < 16; ++j) s += lds[j][lane];
    out[c] = s;
  }
}

constexpr int kNormMaxD = 32768;

// Lanes of a sub-wave team whose chunks cover d (a power of two, 8..64).
int team_log2(int d, int per_lane) {
  int l = 3;
  while (l < 6 && (8 << l) * per_lane < d) ++l;
  return l;
}

int norm_blocks(int T, int teams, int most) {
  return static_cast<int>(std::max(1ll, std::min<long long>((static_cast<long long>(T) + teams - 1) / teams, most)));
}

// As many waves as a row's chunks fill, one chunk a lane up to 4096 columns, two to 16384:
// more waves have more loads in flight (us, against two or four chunks a lane on fewer
// waves: 64 x 2048 bf16 4.8 | 6.2, 8192 x 2048 float32 67 | 76, 4096 x 4096 38.6 | 41.8;
// 8192 x 8192 with one chunk on 16 waves 146, with two on eight 142).  A team takes one
// row: blocks that stay for the next ones wait for theirs (16384 x 4096 128 | 139, 65536 x
// 1024 129 | 142, 8192 x 2112 42 | 51); a grid has fewer than 2^32 threads, so past 2^20
// blocks they do.
template <bool BF16>
void launch_norm(const NormArgs& a, hipStream_t s) {
#define LUFFY_NORM(CH, WAVES)                                                                                    \
  do {                                                                                                           \
    const int lg = team_log2(a.d, CH);                                                                           \
    launch("block_norm", block_norm_kernel<BF16, CH, WAVES>,                                                     \
           norm_blocks(a.T, WAVES > 1 ? 1 : 256 >> lg, 1 << 20), WAVES > 1 ? WAVES * 64 : 256, 0, s, a, lg);     \
  } while (0)
  switch (a.d <= 4096 ? (a.d + 511) / 512 : a.d <= 8192 ? (a.d + 1023) / 1024 + 8 : 0) {
    case 1: LUFFY_NORM(1, 1); break;
    case 2: LUFFY_NORM(1, 2); break;
    case 3: LUFFY_NORM(1, 3); break;
    case 4: LUFFY_NORM(1, 4); break;
    case 5: LUFFY_NORM(1, 5); break;
    case 6: LUFFY_NORM(1, 6); break;
    case 7: LUFFY_NORM(1, 7); break;
    case 8: LUFFY_NORM(1, 8); break;
    case 13: LUFFY_NORM(2, 5); break;
    case 14: LUFFY_NORM(2, 6); break;
    case 15: LUFFY_NORM(2, 7); break;
    case 16: LUFFY_NORM(2, 8); break;
    default:
      if (a.d <= 16384) LUFFY_NORM(2, 16);
      else LUFFY_NORM(4, 16);
  }
#undef LUFFY_NORM
}

// A team of the backward and the blocks of the grid (each leaves kSums rows of d sums
// to be added up).  One chunk a lane on as many waves as a row fills; or two, which halves
// the waves that wait for each other, from 16 rows a team on, where they fill three
// quarters of the lanes (bf16, no bias gradients, us, one | two chunks: 65536 x 1024 207 | 202, 32768 x 2048
// 211 | 199, 16384 x 4096 217 | 199, 8192 x 3520 105 | 99; 8192 x 2880 75 | 90, 8192 x
// 2112 68 | 82, 32768 x 1088 148 | 160; 8192 x 1024 36 | 40; float32 3001 x 1088 33 | 36),
// and, up to 1024 columns, where no bias gradient takes the registers (65536 x 1024 257 |
// 290).
struct BwdShape {
  int chunks, waves, blocks;
};

BwdShape bwd_shape(int T, int d, bool bf16, bool bias) {
  constexpr int most = 256;   // blocks: the workspace is sized without a device
  if (d > 8192) return {d <= 16384 ? 2 : 4, 16, norm_blocks(T, 1, most)};
  if (d > 4096) return {2, 8, norm_blocks(T, 1, most)};
  if (d <= 512) return {1, 1, norm_blocks(T, 512 >> team_log2(d, 1), most)};
  const int two = d <= 1024 ? 1 : d <= 2048 ? 2 : 4, teams = 8 / two;
  if (bf16 && T >= 16 * most * teams && 4 * d > 3 * 1024 * two && !(bias && two == 1))
    return {2, two, norm_blocks(T, teams, most)};
  const int one = (d + 511) / 512;
  return {1, one, norm_blocks(T, bwd_threads(one) / 64 / one, most)};
}

template <bool BF16, bool BIAS>
void launch_norm_backward(const NormBwdArgs& a, float* part, hipStream_t s) {
  const BwdShape sh = bwd_shape(a.T, a.d, BF16, BIAS);
  const int blocks = sh.blocks;
#define LUFFY_NORM_B(CH, WAVES)                                                                           \
  launch("block_norm_backward", block_norm_backward_kernel<BF16, CH, WAVES, BIAS>, blocks,                \
         bwd_threads(WAVES), 0, s, a, team_log2(a.d, CH), part)
  if (sh.waves == 16) {
    if (sh.chunks == 2) LUFFY_NORM_B(2, 16); else LUFFY_NORM_B(4, 16);
  } else if (sh.chunks == 1) {
    if (sh.waves == 1) LUFFY_NORM_B(1, 1);
    else if (sh.waves == 2) LUFFY_NORM_B(1, 2);
    else if (sh.waves == 3) LUFFY_NORM_B(1, 3);
    else if (sh.waves == 4) LUFFY_NORM_B(1, 4);
    else if (sh.waves == 5) LUFFY_NORM_B(1, 5);
    else if (sh.waves == 6) LUFFY_NORM_B(1, 6);
    else if (sh.waves == 7) LUFFY_NORM_B(1, 7);
    else LUFFY_NORM_B(1, 8);
  } else if (sh.waves == 8) {
    LUFFY_NORM_B(2, 8);
  } else if constexpr (BF16) {
    if (sh.waves == 4) LUFFY_NORM_B(2, 4);
    else if (sh.waves == 2) LUFFY_NORM_B(2, 2);
    else if constexpr (!BIAS) LUFFY_NORM_B(2, 1);
  }
#undef LUFFY_NORM_B
  bool any = false;
  for (float* p : a.sum) any = any || p;
  if (any && blocks > 1)
    launch("block_norm_reduce", block_norm_reduce_kernel, dim3(a.d / 64, kSums), 1024, 0, s,
           static_cast<const float*>(part), blocks, a.d, a);
}

// Host checks shared by both directions.
int norm_check(const char* fn, int T, int d, int dtype, int norm, float eps, float res_scale, const void* gate,
               int gate_kind, const void* y, const float* w_post, const float* b_post) {
  if (T <= 0 || d <= 0) return fail(LUFFY_E_INVALID, "%s: T=%d d=%d must be positive", fn, T, d);
  if (dtype != LUFFY_F32 && dtype != LUFFY_BF16) return fail(LUFFY_E_INVALID, "%s: unknown dtype %d", fn, dtype);
  if (norm != LUFFY_NORM_RMS && norm != LUFFY_NORM_LAYER) return fail(LUFFY_E_INVALID, "%s: unknown norm %d", fn, norm);
  if (!(eps >= 0.f)) return fail(LUFFY_E_INVALID, "%s: eps=%g must not be negative", fn, static_cast<double>(eps));
  if (res_scale != res_scale) return fail(LUFFY_E_INVALID, "%s: res_scale is NaN", fn);
  if (gate_kind != LUFFY_GATE_NONE && gate_kind != LUFFY_GATE_CHANNEL && gate_kind != LUFFY_GATE_TOKEN)
    return fail(LUFFY_E_INVALID, "%s: unknown gate kind %d", fn, gate_kind);
  if ((gate != nullptr) != (gate_kind != LUFFY_GATE_NONE))
    return fail(LUFFY_E_INVALID, "%s: gate kind %d with gate %p", fn, gate_kind, gate);
  if (!y && (w_post || b_post || gate || res_scale != 1.0f))
    return fail(LUFFY_E_INVALID, "%s: w_post, b_post, gate and res_scale belong to y, which is null", fn);
  if (b_post && !w_post) return fail(LUFFY_E_INVALID, "%s: b_post without w_post", fn);
  if (d % 64 != 0) return fail(LUFFY_E_UNSUPPORTED, "%s: d=%d not a multiple of 64", fn, d);
  if (d > kNormMaxD) return fail(LUFFY_E_UNSUPPORTED, "%s: d=%d > %d", fn, d, kNormMaxD);
  if (T > (1 << 30)) return fail(LUFFY_E_UNSUPPORTED, "%s: T=%d > 2^30", fn, T);
  return LUFFY_OK;
}

bool aligned16(std::initializer_list<const void*> ps) {
  uintptr_t bits = 0;
  for (const void* p : ps) bits |= reinterpret_cast<uintptr_t>(p);
  return (bits & 15u) == 0;
}

}  // namespace
}  // namespace luffy

using namespace luffy;

extern "C" int luffy_block_norm(const void* x, const void* y, int T, int d, int dtype, int norm, float eps,
                                const float* w_post, const float* b_post, const void* gate, int gate_kind,
                                float res_scale, const float* w_pre, const float* b_pre, void* o, void* u,
                                void* stream) {
  const char* fn = "luffy_block_norm";
  if (!x) return fail(LUFFY_E_INVALID, "%s: x is null", fn);
  if ((y != nullptr) != (o != nullptr)) return fail(LUFFY_E_INVALID, "%s: o is written where y is given", fn);
  if ((w_pre != nullptr) != (u != nullptr)) return fail(LUFFY_E_INVALID, "%s: u is written where w_pre is given", fn);
  if (b_pre && !w_pre) return fail(LUFFY_E_INVALID, "%s: b_pre without w_pre", fn);
  if (!o && !u) return fail(LUFFY_E_INVALID, "%s: neither o nor u", fn);
  const int st = norm_check(fn, T, d, dtype, norm, eps, res_scale, gate, gate_kind, y, w_post, b_post);
  if (st != LUFFY_OK) return st;
  if (!aligned16({x, y, w_post, b_post, gate, w_pre, b_pre, o, u}))
    return fail(LUFFY_E_INVALID, "%s: a pointer is not 16-byte aligned", fn);
  const NormArgs a{x, y, w_post, b_post, w_pre, b_pre, gate, gate_kind, T, d, norm == LUFFY_NORM_LAYER, eps,
                   res_scale, o, u};
  if (dtype == LUFFY_BF16) launch_norm<true>(a, static_cast<hipStream_t>(stream));
  else launch_norm<false>(a, static_cast<hipStream_t>(stream));
  return check_launch(fn);
}

extern "C" size_t luffy_block_norm_backward_workspace_size(int T, int d) {
  if (T <= 0 || d <= 0) return 0;
  Carver c(nullptr);
  int blocks = 0;   // of any type and any gradients
  for (const bool bf16 : {false, true})
    for (const bool bias : {false, true}) blocks = std::max(blocks, bwd_shape(T, d, bf16, bias).blocks);
  c.take<float>(static_cast<size_t>(blocks) * kSums * d);
  return c.size();
}

extern "C" int luffy_block_norm_backward(const void* y, const void* o, int T, int d, int dtype, int norm, float eps,
                                         const float* w_post, const float* b_post, const void* gate, int gate_kind,
                                         float res_scale, const float* w_pre, const void* dout, const void* du,
                                         void* dx, void* dy, void* dgate, float* dw_post, float* db_post,
                                         float* dw_pre, float* db_pre, void* workspace, size_t workspace_bytes,
                                         void* stream) {
  const char* fn = "luffy_block_norm_backward";
  if (!dx) return fail(LUFFY_E_INVALID, "%s: dx is null", fn);
  if (!dout && !du) return fail(LUFFY_E_INVALID, "%s: neither do nor du", fn);
  if (du && (!w_pre || !o)) return fail(LUFFY_E_INVALID, "%s: du needs o and w_pre", fn);
  if ((y != nullptr) != (dy != nullptr)) return fail(LUFFY_E_INVALID, "%s: dy is written where y is given", fn);
  if (!du && (dw_pre || db_pre)) return fail(LUFFY_E_INVALID, "%s: dw_pre and db_pre need du", fn);
  if (!w_post && (dw_post || db_post)) return fail(LUFFY_E_INVALID, "%s: dw_post and db_post need w_post", fn);
  if (!gate && dgate) return fail(LUFFY_E_INVALID, "%s: dgate without a gate", fn);
  const int st = norm_check(fn, T, d, dtype, norm, eps, res_scale, gate, gate_kind, y, w_post, b_post);
  if (st != LUFFY_OK) return st;
  if (!aligned16({y, o, w_post, b_post, gate, w_pre, dout, du, dx, dy, dgate, dw_post, db_post, dw_pre, db_pre}))
    return fail(LUFFY_E_INVALID, "%s: a pointer is not 16-byte aligned", fn);
  const size_t need = luffy_block_norm_backward_workspace_size(T, d);
  if (workspace_bytes < need || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return fail(LUFFY_E_WORKSPACE, "%s: workspace needs %zu bytes, 256-aligned", fn, need);
  NormBwdArgs a{y, o, dout, du, w_post, b_post, w_pre, gate, gate_kind, T, d, norm == LUFFY_NORM_LAYER, eps, res_scale,
                dx, dy, gate_kind == LUFFY_GATE_TOKEN ? dgate : nullptr, {}};
  a.sum[0] = dw_pre;
  a.sum[1] = db_pre;
  a.sum[2] = dw_post;
  a.sum[3] = db_post;
  a.sum[4] = gate_kind == LUFFY_GATE_CHANNEL ? static_cast<float*>(dgate) : nullptr;
  const bool bias = db_pre || db_post;
  auto* run = dtype == LUFFY_BF16 ? (bias ? launch_norm_backward<true, true> : launch_norm_backward<true, false>)
                                  : (bias ? launch_norm_backward<false, true> : launch_norm_backward<false, false>);
  run(a, static_cast<float*>(workspace), static_cast<hipStream_t>(stream));
  return check_launch(fn);
}
