// Y = act(W X + bias) + R: projections of a decoder layer.
#include "linear.h"

namespace strp {

// Products of fp32 (v_mfma_f32_32x32x2_f32: an operand of bf16 is widened, which is exact).  Tiles of 128 channels x 128 tokens,
// four wavefronts of 64 x 64, 16 contraction steps in LDS while the next 16 are on their way to registers.  Rows of X and columns
// of W from K on are zeros in LDS, whatever memory holds there.
template <typename WT, typename XT, typename YT>
__global__ __launch_bounds__(256) void linear_f32_kernel(const LinearP p) {
  constexpr int BM = 128, BN = 128, BK = 16, PAD = 4;
  __shared__ float sW[BK][BM + PAD], sX[BK][BN + PAD];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = lane >> 5, l32 = lane & 31;
  const int m0 = (int)(blockIdx.x % p.tilesM) * BM;
  const long long n0 = (long long)(blockIdx.x / p.tilesM) * BN;
  const int wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
  const int wr = tid >> 2, wk = (tid & 3) * 4;          // W: row wr (+ 64), columns wk .. wk + 3 of the step
  const int xr = tid >> 5, xt = (tid & 31) * 4;         // X: row xr (+ 8), tokens xt .. xt + 3
  float w[2][4], x[2][4];
  auto fetch = [&](int k0) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int m = m0 + wr + 64 * i, k = k0 + wk;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[i][e] = x[i][e] = 0.0f;
      if (m < p.M && k < p.K) {
        load_floats<4>((const WT*)p.W + (long long)m * p.ldw + k, w[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[i][e] = k + e < p.K ? w[i][e] : 0.0f;
      }
      const int kx = k0 + xr + 8 * i;
      if (kx < p.K && n0 + xt < p.T) load_floats<4>((const XT*)p.X + (long long)kx * p.ldx + n0 + xt, x[i]);
    }
  };
  floatx16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
  fetch(0);
  for (int k0 = 0; k0 < p.K; k0 += BK) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int e = 0; e < 4; ++e) sW[wk + e][wr + 64 * i] = w[i][e];
      *(floatx4*)&sX[xr + 8 * i][xt] = floatx4{x[i][0], x[i][1], x[i][2], x[i][3]};
    }
    __syncthreads();
    if (k0 + BK < p.K) fetch(k0 + BK);
#pragma unroll
    for (int s = 0; s < BK / 2; ++s) {
      float a[2], b[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        a[i] = sW[2 * s + h][wm + 32 * i + l32];
        b[i] = sX[2 * s + h][wn + 32 * i + l32];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[j], acc[i][j], 0, 0, 0);
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int m = m0 + wm + 32 * i + 8 * (e >> 2) + 4 * h + (e & 3);
        const long long t = n0 + wn + 32 * j + l32;
        if (m >= p.M || t >= p.T) continue;
        float y = activate(acc[i][j][e] + (p.bias ? p.bias[m] : 0.0f), p.act);
        if (p.R) y += (float)((const YT*)p.R)[(long long)m * p.ldr + t];
        ((YT*)p.Y)[(long long)m * p.ldy + t] = (YT)y;
      }
}

template <typename WT, typename XT>
static void launch_linear_f32(strp_ctx* ctx, LinearP& p, int y_dtype) {
  p.tilesM = (p.M + 127) / 128;
  const dim3 grid((unsigned)(p.tilesM * ((p.T + 127) / 128))), block(256);
  if (y_dtype == STRP_BF16) hipLaunchKernelGGL((linear_f32_kernel<WT, XT, __bf16>), grid, block, 0, ctx->stream, p);
  else hipLaunchKernelGGL((linear_f32_kernel<WT, XT, float>), grid, block, 0, ctx->stream, p);
}

}  // namespace strp

using namespace strp;

extern "C" {

size_t strp_linear_workspace_bytes(int32_t M, int32_t K, int64_t T, strp_dtype w_dtype, strp_dtype x_dtype) {
  if (M <= 0 || K <= 0 || T <= 0) return 0;
  if (w_dtype != STRP_BF16 || x_dtype != STRP_BF16) return 0;
  const size_t part = plan_linear_bf16(M, K, T).part_bytes;
  return part ? part + 4096 : 0;
}

strp_status strp_linear(strp_ctx* ctx, const strp_linear_in* in) {
  if (!ctx) return STRP_EINVAL;
  if (!in || !in->W || !in->X || !in->Y) return fail(ctx, STRP_EINVAL, "linear: null W, X or Y");
  if (!known_dtype(in->w_dtype) || !known_dtype(in->x_dtype) || !known_dtype(in->y_dtype)) return fail(ctx, STRP_EINVAL, "linear: unknown dtype");
  if (in->M <= 0 || in->K <= 0 || in->T <= 0) return fail(ctx, STRP_EINVAL, "linear: M, K, T must be positive");
  if (in->act != STRP_ACT_NONE && in->act != STRP_ACT_RELU && in->act != STRP_ACT_GELU) return fail(ctx, STRP_EINVAL, "linear: unknown activation");
  if (!token_ld(in->ldx, in->T) || !token_ld(in->ldy, in->T) || (in->R && !token_ld(in->ldr, in->T)) || !token_ld(in->ldw, in->K))
    return fail(ctx, STRP_EINVAL, "linear: leading dimensions must be multiples of 8 and not below T (ldw: K)");
  if (!ptr16(in->W) || !ptr16(in->X) || !ptr16(in->Y) || !ptr16(in->R)) return fail(ctx, STRP_EINVAL, "linear: W, X, R or Y not 16-byte aligned");
  if (in->R == in->Y && in->ldr != in->ldy) return fail(ctx, STRP_EINVAL, "linear: R is Y with another leading dimension");
  if ((in->M + 63) / 64 * ((in->T + 63) / 64) > 0x7fffffffLL) return fail(ctx, STRP_EINVAL, "linear: more than 2^31 tiles of 64 x 64");
  LinearP p{in->W, in->X, in->bias, in->R, in->Y, in->M, in->K, in->act, in->T, in->ldw, in->ldx, in->ldr, in->ldy};
  p.splits = 1;
  LinearPlan plan{};
  const int wb = in->w_dtype == STRP_BF16, xb = in->x_dtype == STRP_BF16;
  if (wb && xb) {
    plan = plan_linear_bf16(p.M, p.K, p.T);
    if (plan.part_bytes) {
      if (!ctx->ws) return fail(ctx, STRP_ENOMEM, "linear: no workspace set");
      Arena arena(ctx);
      STRP_TAKE(ctx, arena, part, float, plan.part_bytes / 4);
      p.part = part;
    }
  }
  OnDevice on(ctx);
  if (!on.ok()) return fail(ctx, STRP_EHIP, "linear: device %d cannot be made current", ctx->device);
  const double M = in->M, K = in->K, T = (double)in->T;
  ProfScope ps(ctx, "linear", 2.0 * M * K * T, bytes_of(in->w_dtype) * M * K + bytes_of(in->x_dtype) * K * T + bytes_of(in->y_dtype) * M * T * (in->R ? 2 : 1));
  if (wb && xb) launch_linear_bf16(ctx, p, plan, in->y_dtype);
  else if (wb) launch_linear_f32<__bf16, float>(ctx, p, in->y_dtype);
  else if (xb) launch_linear_f32<float, __bf16>(ctx, p, in->y_dtype);
  else launch_linear_f32<float, float>(ctx, p, in->y_dtype);
  STRP_HIP(ctx, hipGetLastError());
  return STRP_OK;
}

}  // extern "C"
