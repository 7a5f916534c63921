// A gated feed-forward block's up-projections, activation and product for a few
// tokens (serving): [g | u] = y Wgu^T + b, h = act(g) u, of up to 32 rows.
//
// Bound by reading the weights once.  Each workgroup takes 8 columns of F: their
// gate and up-projection rows are the 16 rows of the A operand of
// v_mfma_f32_16x16x32_bf16 (by 16 tokens).  Its waves share the contraction, 64
// columns at a time, so that together they read whole lines of each row, straight
// into registers, with kAhead 64-wide steps in flight per wave; the tokens'
// operand comes from the caches.  The waves' fp32 sums are added in LDS in wave
// order, then bias, activation and product follow: one launch, no workspace.
// One token, us (TB/s of weights), against the tiled product and its split's
// second launch: 1280 x 3416 6.0 (2.9) / 15.4, 6144 x 2048 12.0 (4.2) / 20.5,
// 6144 x 16384 71 (5.7) / 75-92.
#include "common.hpp"
#include "gate.hpp"
#include "kernels.hpp"

namespace optimus {

namespace {

constexpr int kCols = 8, kWaves = 8, kAhead = 4;

template <int NB>  // 16 tokens each
__global__ __launch_bounds__(64 * kWaves) void glu_small_kernel(int M, int F, int K, int act,
                                                                const bf16_t *__restrict__ y,
                                                                const bf16_t *__restrict__ w,
                                                                const bf16_t *__restrict__ bias,
                                                                bf16_t *__restrict__ gu, bf16_t *__restrict__ h) {
  __shared__ f32x4_t part[kWaves][NB][64];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int j0 = blockIdx.x * kCols, r = lane & 15, kl = (lane >> 4) * 8;
  // (F is a multiple of 8: every column of the workgroup exists)
  const bf16_t *wr = w + static_cast<size_t>(j0 + (r & 7) + (r >= 8 ? F : 0)) * K;
  const u32x4_t zero{0u, 0u, 0u, 0u};
  const int steps = (K + 63) / 64;
  f32x4_t acc[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) acc[n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int s0 = wid; s0 < steps; s0 += kWaves * kAhead) {
    u32x4_t a[kAhead][2], b[kAhead][2][NB];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int k = (s0 + i * kWaves) * 64 + e * 32 + kl;
        const bool in = k < K;  // (K is a multiple of 8)
        a[i][e] = in ? ldg16(wr + k) : zero;
#pragma unroll
        for (int n = 0; n < NB; ++n)
          b[i][e][n] = in && 16 * n + r < M ? ldg16(y + static_cast<size_t>(16 * n + r) * K + k) : zero;
      }
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[n] = mfma16(as_bf16x8(a[i][e]), as_bf16x8(b[i][e][n]), acc[n]);
  }
#pragma unroll
  for (int n = 0; n < NB; ++n) part[wid][n][lane] = acc[n];
  __syncthreads();
  // lanes 0..31 of a result hold four gates of token lane % 16, lanes 32..63
  // the same columns' up-projections
  if (threadIdx.x < 32 * NB) {
    const int n = lane >> 5, l = lane & 31;
    f32x4_t gs = part[0][n][l], us = part[0][n][l + 32];
#pragma unroll
    for (int s = 1; s < kWaves; ++s) gs += part[s][n][l], us += part[s][n][l + 32];
    const int m = 16 * n + r, j = j0 + (l >> 4) * 4;
    if (m >= M) return;
    float gv[4], uv[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      gv[e] = gs[e] + (bias ? bf2f(bias[j + e]) : 0.f);
      uv[e] = us[e] + (bias ? bf2f(bias[F + j + e]) : 0.f);
    }
    if (gu) {
      bf16_t *o = gu + static_cast<size_t>(m) * 2 * F + j;
      *reinterpret_cast<u32x2_t *>(o) = u32x2_t{pack2(gv[0], gv[1]), pack2(gv[2], gv[3])};
      *reinterpret_cast<u32x2_t *>(o + F) = u32x2_t{pack2(uv[0], uv[1]), pack2(uv[2], uv[3])};
    }
    *reinterpret_cast<u32x2_t *>(h + static_cast<size_t>(m) * F + j) =
        u32x2_t{pack2(gate_f(gv[0], act) * uv[0], gate_f(gv[1], act) * uv[1]),
                pack2(gate_f(gv[2], act) * uv[2], gate_f(gv[3], act) * uv[3])};
  }
}

}  // namespace

bool launch_glu_small(int M, int F, int K, int act, const bf16_t *y, const bf16_t *w, const bf16_t *bias, bf16_t *gu,
                      bf16_t *h, hipStream_t s) {
  hipLaunchKernelGGL(M <= 16 ? glu_small_kernel<1> : glu_small_kernel<2>, dim3(F / kCols), dim3(64 * kWaves), 0, s, M, F,
                     K, act, y, w, bias, gu, h);
  return true;
}

}  // namespace optimus
