// Layer normalisation over the channels of every token, channel-major.
#include "layer_ops.h"

namespace strp {

struct NormP {
  const void* X;
  void* Y;
  const float* gain;
  const float* bias;
  int d;
  long long T, ldx, ldy;
  float eps;
};

// A workgroup has eight 16-byte columns of tokens and reads their rows 32 at a time, three times: mean, mean square of the
// deviations, result.
template <typename E>
__global__ __launch_bounds__(256) void layer_norm_kernel(const NormP p) {
  constexpr int VEC = 16 / sizeof(E), CT = 8, RL = 32;
  __shared__ float sh[RL][CT * VEC + 1];
  const int c = threadIdx.x % CT, r = threadIdx.x / CT;
  const long long t0 = ((long long)blockIdx.x * CT + c) * VEC;
  const bool in = t0 < p.T;
  const E* x = (const E*)p.X + t0;
  E* y = (E*)p.Y + t0;
  // sums over the row lanes, in every thread of a column, always in the same order
  auto total = [&](float (&v)[VEC]) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < VEC; ++e) sh[r][c * VEC + e] = v[e];
    __syncthreads();
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      float a = 0.0f;
      for (int i = 0; i < RL; ++i) a += sh[i][c * VEC + e];
      v[e] = a;
    }
  };
  float mean[VEC], rs[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) mean[e] = rs[e] = 0.0f;
  if (in)
    for (int j = r; j < p.d; j += RL) {
      float v[VEC];
      load_floats<VEC>(x + (long long)j * p.ldx, v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) mean[e] += v[e];
    }
  total(mean);
#pragma unroll
  for (int e = 0; e < VEC; ++e) mean[e] /= (float)p.d;
  if (in)
    for (int j = r; j < p.d; j += RL) {
      float v[VEC];
      load_floats<VEC>(x + (long long)j * p.ldx, v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) rs[e] += (v[e] - mean[e]) * (v[e] - mean[e]);
    }
  total(rs);
#pragma unroll
  for (int e = 0; e < VEC; ++e) rs[e] = 1.0f / sqrtf(rs[e] / (float)p.d + p.eps);
  if (!in) return;
  for (int j = r; j < p.d; j += RL) {
    float v[VEC];
    load_floats<VEC>(x + (long long)j * p.ldx, v);
    const float g = p.gain ? p.gain[j] : 1.0f, b = p.bias ? p.bias[j] : 0.0f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = (v[e] - mean[e]) * rs[e] * g + b;
    if (t0 + VEC <= p.T) store_floats<VEC>(y + (long long)j * p.ldy, v);
    else
      for (int e = 0; e < VEC; ++e)
        if (t0 + e < p.T) y[(long long)j * p.ldy + e] = (E)v[e];
  }
}

}  // namespace strp

using namespace strp;

extern "C" strp_status strp_layer_norm(strp_ctx* ctx, const void* X, strp_dtype dtype, int32_t d, int64_t T, int64_t ldx, const float* gain,
                                       const float* bias, double eps, void* Y, int64_t ldy) {
  if (!ctx) return STRP_EINVAL;
  if (!X || !Y) return fail(ctx, STRP_EINVAL, "layer_norm: null X or Y");
  if (!known_dtype(dtype)) return fail(ctx, STRP_EINVAL, "layer_norm: unknown dtype");
  if (d <= 0 || T <= 0) return fail(ctx, STRP_EINVAL, "layer_norm: d and T must be positive");
  if (!(eps >= 0.0)) return fail(ctx, STRP_EINVAL, "layer_norm: eps must not be negative");
  if (!token_ld(ldx, T) || !token_ld(ldy, T)) return fail(ctx, STRP_EINVAL, "layer_norm: leading dimensions must be multiples of 8 and not below T");
  if (!ptr16(X) || !ptr16(Y)) return fail(ctx, STRP_EINVAL, "layer_norm: X or Y not 16-byte aligned");
  if (X == Y && ldx != ldy) return fail(ctx, STRP_EINVAL, "layer_norm: Y is X with another leading dimension");
  if (T > (1LL << 34)) return fail(ctx, STRP_EINVAL, "layer_norm: more than 2^34 tokens");
  OnDevice on(ctx);
  if (!on.ok()) return fail(ctx, STRP_EHIP, "layer_norm: device %d cannot be made current", ctx->device);
  const NormP p{X, Y, gain, bias, d, T, ldx, ldy, (float)eps};
  ProfScope ps(ctx, "layer_norm", 7.0 * d * (double)T, 2.0 * bytes_of(dtype) * d * (double)T);
  const long long cols = 128 / (long long)bytes_of(dtype);
  const dim3 grid((unsigned)((T + cols - 1) / cols)), block(256);
  if (dtype == STRP_BF16) hipLaunchKernelGGL((layer_norm_kernel<__bf16>), grid, block, 0, ctx->stream, p);
  else hipLaunchKernelGGL((layer_norm_kernel<float>), grid, block, 0, ctx->stream, p);
  STRP_HIP(ctx, hipGetLastError());
  return STRP_OK;
}
