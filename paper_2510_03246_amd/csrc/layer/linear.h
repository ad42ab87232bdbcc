// The products of strp_linear: what the entry point hands to the kernels.
#pragma once

#include "layer_ops.h"

namespace strp {

struct LinearP {
  const void* W;
  const void* X;
  const float* bias;
  const void* R;
  void* Y;
  int M, K, act;
  long long T, ldw, ldx, ldr, ldy;
  int tilesM, tilesN;
  int splits, pairs;     // parts of the contraction and pairs of steps of 32 of each; more than one part: sums to part, [splits][M][tp]
  float* part;
  long long tp;
};

__device__ __forceinline__ float activate(float z, int act) {
  if (act == STRP_ACT_RELU) return z > 0.0f ? z : (z == z ? 0.0f : z);
  // z Phi(z) with Phi from the complementary error function: no cancellation where z is far below zero
  if (act == STRP_ACT_GELU) return 0.5f * z * erfcf(-0.70710678118654752f * z);
  return z;
}

// Bias, activation and residual on the sums v of four tokens from t on, channel m; t < T, m < M.
template <typename YT>
__device__ __forceinline__ void finish_quad(const LinearP& p, floatx4 v, int m, long long t) {
  float y[4], r[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  if (p.R) load_floats<4>((const YT*)p.R + (long long)m * p.ldr + t, r);
  const float b = p.bias ? p.bias[m] : 0.0f;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = activate(v[e] + b, p.act) + r[e];
  YT* Y = (YT*)p.Y + (long long)m * p.ldy + t;
  if (t + 4 <= p.T) store_floats<4>(Y, y);
  else
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (t + e < p.T) Y[e] = (YT)y[e];
}

// How a product is cut, by sizes and types only: tile shape, parts of the contraction.  kind: of products of bf16.
enum { LINEAR_FEW, LINEAR_TILE_SMALL, LINEAR_TILE, LINEAR_TILE_LARGE };
struct LinearPlan {
  int kind;
  int bm, bn;
  int splits, pairs;
  size_t part_bytes;
};
LinearPlan plan_linear_bf16(int M, int K, long long T);
void launch_linear_bf16(strp_ctx* ctx, LinearP p, const LinearPlan& plan, int y_dtype);
// sums of the parts, bias, activation, residual
void launch_linear_join(strp_ctx* ctx, const LinearP& p, int y_dtype);

}  // namespace strp
