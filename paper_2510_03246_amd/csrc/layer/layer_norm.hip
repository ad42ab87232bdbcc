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
  int ct;
};

__device__ __forceinline__ float norm_shift(float v, float mean, float rs, float g, float b) { return (v - mean) * rs * g + b; }

template <int CTL>
__device__ __forceinline__ float lanes_by(float a) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, a), CTL, 0xf, 0xf, false));
}
// the sum of the four rows of 16 lanes, in each of them
__device__ __forceinline__ float all_rows(float a) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, a), false, false);
  const unsigned r0 = r[0], r1 = r[1];
  const float b = __builtin_bit_cast(float, r0) + __builtin_bit_cast(float, r1);
  const auto h = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, b), __builtin_bit_cast(unsigned, b), false, false);
  const unsigned h0 = h[0], h1 = h[1];
  return __builtin_bit_cast(float, h0) + __builtin_bit_cast(float, h1);
}

// A workgroup has ct columns of 16 bytes (a power of two) and all their rows in registers, NR to a thread: memory is read once and written once, which is what
// bounds it, with one workgroup on a CU.  Both sums, of the values and of the squares of their deviations from the mean, are over what is in registers.  bf16: 4096 channels over 32768 tokens 164 to 174 us,
// 3.1 to 3.2 TB/s (over 8192, from and to the last-level cache, 30 us, 4.4); 7168 over 32768 382 us, 2.5; 768 over 2048 8.2 us, latencies.
template <typename E, int NR>
__global__ __launch_bounds__(1024) void layer_norm_kernel(const NormP p) {
  constexpr int VEC = 16 / sizeof(E);
  __shared__ __attribute__((aligned(16))) float part[16][16 * VEC], whole[16 * VEC];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = tid & (p.ct - 1), bits = 31 - __clz(p.ct), r0 = tid >> bits, rl = 1024 >> bits;
  // workgroups go to the eight XCDs in turn: the g neighbours that share a line of memory go to one, and those that run at a time still lie side by side
  const unsigned g = p.ct < 8 ? 8 / p.ct : 1, b0 = blockIdx.x / (8 * g) * (8 * g), in_g = blockIdx.x - b0;
  const long long at = b0 + 8 * g <= gridDim.x ? b0 + (in_g & 7) * g + (in_g >> 3) : blockIdx.x;
  const long long t0 = (at * p.ct + c) * VEC;
  const bool in = t0 < p.T;
  const E* x = (const E*)p.X + (in ? t0 : 0);
  E* y = (E*)p.Y + t0;
  uintx4 v[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const int j = r0 + i * rl;
    v[i] = uintx4{0u, 0u, 0u, 0u};
    if (j < p.d) v[i] = *(const uintx4*)(x + (long long)j * p.ldx);
  }
  // asked for early where there are registers for it
  constexpr int EARLY = NR <= 4 ? NR : 1;
  float gain[EARLY], bias[EARLY];
  if (NR <= 4)
#pragma unroll
    for (int i = 0; i < EARLY; ++i) {
      const int j = min(r0 + i * rl, p.d - 1);
      gain[i] = p.gain ? p.gain[j] : 1.0f;
      bias[i] = p.bias ? p.bias[j] : 0.0f;
    }
  typedef E vec __attribute__((ext_vector_type(VEC)));
  // sums over a column's threads, in each of them: the wavefront's by exchange, the workgroup's through LDS, in one order
  auto total = [&](float (&a)[VEC]) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      if (p.ct <= 1) a[e] += lanes_by<0xb1>(a[e]);        // neighbours, pairs, then 4 and 8 lanes round a row of 16
      if (p.ct <= 2) a[e] += lanes_by<0x4e>(a[e]);
      if (p.ct <= 4) a[e] += lanes_by<0x124>(a[e]);
      if (p.ct <= 8) a[e] += lanes_by<0x128>(a[e]);
      a[e] = all_rows(a[e]);
    }
    if (lane < p.ct)
#pragma unroll
      for (int e = 0; e < VEC; ++e) part[wave][c * VEC + e] = a[e];
    __syncthreads();
    if (tid < p.ct * VEC) {
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < 16; ++w) s += part[w][tid];
      whole[tid] = s;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < VEC; ++e) a[e] = whole[c * VEC + e];
  };
  // the values as they were read, not as floats, go from one pass over them to the next
  auto keep = [&]() {
#pragma unroll
    for (int i = 0; i < NR; ++i) asm volatile("" : "+v"(v[i]));
  };
  float mean[VEC], rs[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) mean[e] = rs[e] = 0.0f;
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const vec f = __builtin_bit_cast(vec, v[i]);
#pragma unroll
    for (int e = 0; e < VEC; ++e) mean[e] += (float)f[e];
  }
  total(mean);
  keep();
#pragma unroll
  for (int e = 0; e < VEC; ++e) mean[e] /= (float)p.d;
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const vec f = __builtin_bit_cast(vec, v[i]);
    if (r0 + i * rl < p.d)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float dev = (float)f[e] - mean[e];
        rs[e] += dev * dev;
      }
  }
  total(rs);
  keep();
#pragma unroll
  for (int e = 0; e < VEC; ++e) rs[e] = 1.0f / sqrtf(rs[e] / (float)p.d + p.eps);
  if (!in) return;
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const int j = r0 + i * rl;
    if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);
    if (j >= p.d) continue;
    const float g1 = NR <= 4 ? gain[NR <= 4 ? i : 0] : (p.gain ? p.gain[j] : 1.0f), b1 = NR <= 4 ? bias[NR <= 4 ? i : 0] : (p.bias ? p.bias[j] : 0.0f);
    const vec f = __builtin_bit_cast(vec, v[i]);
    float o[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) o[e] = norm_shift((float)f[e], mean[e], rs[e], g1, b1);
    if (t0 + VEC <= p.T) store_floats<VEC>(y + (long long)j * p.ldy, o);
    else
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (t0 + e < p.T) y[(long long)j * p.ldy + e] = (E)o[e];
  }
}

// The same for more rows than registers hold: a workgroup reads its columns three times, for the mean, the deviations and the result.
template <typename E>
__global__ __launch_bounds__(256) void layer_norm_tall_kernel(const NormP p) {
  constexpr int VEC = 16 / sizeof(E), CT = 8, RL = 32;
  __shared__ float sh[RL][CT * VEC + 1];
  const int c = threadIdx.x % CT, r = threadIdx.x / CT;
  const long long t0 = ((long long)blockIdx.x * CT + c) * VEC;
  const bool in = t0 < p.T;
  const E* x = (const E*)p.X + (in ? t0 : 0);
  E* y = (E*)p.Y + t0;
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
#pragma unroll 4
  for (int j = r; j < p.d; j += RL) {
    float v[VEC];
    load_floats<VEC>(x + (long long)j * p.ldx, v);
#pragma unroll
    for (int e = 0; e < VEC; ++e) mean[e] += v[e];
  }
  total(mean);
#pragma unroll
  for (int e = 0; e < VEC; ++e) mean[e] /= (float)p.d;
#pragma unroll 4
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
#pragma unroll 4
  for (int j = r; j < p.d; j += RL) {
    float v[VEC];
    load_floats<VEC>(x + (long long)j * p.ldx, v);
    const float g = p.gain ? p.gain[j] : 1.0f, b = p.bias ? p.bias[j] : 0.0f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = norm_shift(v[e], mean[e], rs[e], g, b);
    if (t0 + VEC <= p.T) store_floats<VEC>(y + (long long)j * p.ldy, v);
    else
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (t0 + e < p.T) y[(long long)j * p.ldy + e] = (E)v[e];
  }
}

template <typename E>
static void launch_norm(strp_ctx* ctx, NormP p) {
  constexpr long long VEC = 16 / sizeof(E);
  const long long chunks = (p.T + VEC - 1) / VEC;
  const auto go = [&](auto kernel, long long cols, int threads) { hipLaunchKernelGGL(kernel, dim3((unsigned)((chunks + cols - 1) / cols)), dim3(threads), 0, ctx->stream, p); };
  // As wide a piece of a row as sixteen rows to a thread hold, narrower where that leaves CUs without work (us, bf16): 768 channels over 65536 tokens in 16 columns 48, 8 57,
  // 4 61; 768 over 8192 in 16 17, 8 13.7, 4 12.1, 2 15.7; 2048 over 16384 in 8 28.7, 4 34.7; 768 over 2048 in 4 9.1, 2 8.3, 1 8.4; 2048 over 2048 in 4 13.2, 2 11.0.
  int ct = 16;
  while (ct > 1 && ((long long)p.d * ct > 16 * 1024 || (ct > 4 && chunks / ct < 256) || chunks / ct < 128)) ct >>= 1;
  const long long rows = ((long long)p.d * ct + 1023) / 1024;
  p.ct = ct;
  if (rows > 16) return go(layer_norm_tall_kernel<E>, 8, 256);
  if (rows <= 2) go(layer_norm_kernel<E, 2>, ct, 1024);
  else if (rows <= 4) go(layer_norm_kernel<E, 4>, ct, 1024);
  else if (rows <= 8) go(layer_norm_kernel<E, 8>, ct, 1024);
  else go(layer_norm_kernel<E, 16>, ct, 1024);
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
  if (T > (1LL << 27) || d > (1 << 30)) return fail(ctx, STRP_EINVAL, "layer_norm: more than 2^27 tokens or 2^30 channels");
  OnDevice on(ctx);
  if (!on.ok()) return fail(ctx, STRP_EHIP, "layer_norm: device %d cannot be made current", ctx->device);
  const NormP p{X, Y, gain, bias, d, T, ldx, ldy, (float)eps, 0};
  ProfScope ps(ctx, "layer_norm", 7.0 * d * (double)T, 2.0 * bytes_of(dtype) * d * (double)T);
  if (dtype == STRP_BF16) launch_norm<__bf16>(ctx, p);
  else launch_norm<float>(ctx, p);
  STRP_HIP(ctx, hipGetLastError());
  return STRP_OK;
}
