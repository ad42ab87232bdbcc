// Y = act(W X + bias) + R: projections of a decoder layer.
#include "linear.h"

namespace strp {

// Products of fp32 (v_mfma_f32_16x16x4_f32: an operand of bf16 is widened, which is exact).  Tiles of BM channels x BN tokens, four wavefronts of a quarter each, 32
// contraction steps in LDS, the next 32 on their way there and those behind them to registers.  Rows of X and columns of W from K on are zeros in LDS, whatever memory holds there.
// What bounds it is the matrix cores (154 TFLOP/s on a large library product), and with few tiles how evenly they go onto the CUs.
template <int BM, int BN, typename WT, typename XT, typename YT>
__global__ __launch_bounds__(256, 2) void linear_f32_kernel(const LinearP p) {
  constexpr int BK = 32, PAD = 20, NI = BM / 32, NJ = BN / 32, RW = BM / 32, RX = BK * BN / 1024, XROWS = 1024 / BN;
  __shared__ __attribute__((aligned(16))) float sW[2][BK][BM + PAD], sX[2][BK][BN + PAD];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, kq = lane >> 4, l16 = lane & 15;
  const int tiles = p.tilesM * p.tilesN, split = (int)blockIdx.x / tiles, tile = (int)blockIdx.x - split * tiles;
  const int m0 = tile % p.tilesM * BM;
  const long long n0 = (long long)(tile / p.tilesM) * BN;
  const int wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);
  const int k_first = split * p.pairs * 64, k_end = min(p.K, k_first + p.pairs * 64);
  const int wr = tid >> 3, wk = (tid & 7) * 4;                     // W: row wr (+ 32 i), columns wk .. wk + 3 of the step
  const int xr = tid / (BN / 4), xt = tid % (BN / 4) * 4;          // X: row xr (+ XROWS i), tokens xt .. xt + 3
  // as they are read: anything done to them here would wait for them
  typedef WT wvec __attribute__((ext_vector_type(4)));
  typedef XT xvec __attribute__((ext_vector_type(4)));
  wvec w[RW];
  xvec x[RX];
  // rows behind M and tokens behind T are others over again: what comes of them is not stored
  const WT* wp[RW];
  const XT* xp[RX];
#pragma unroll
  for (int i = 0; i < RW; ++i) wp[i] = (const WT*)p.W + (long long)min(m0 + wr + 32 * i, p.M - 1) * p.ldw + wk;
#pragma unroll
  for (int i = 0; i < RX; ++i) xp[i] = (const XT*)p.X + (long long)(xr + XROWS * i) * p.ldx + (n0 + xt < p.T ? n0 + xt : (p.T - 1) / 4 * 4);
  auto fetch = [&](int k0) {
    if (k0 + BK <= k_end) {
#pragma unroll
      for (int i = 0; i < RW; ++i) w[i] = *(const wvec*)(wp[i] + k0);
#pragma unroll
      for (int i = 0; i < RX; ++i) x[i] = *(const xvec*)(xp[i] + (long long)k0 * p.ldx);
    } else {
#pragma unroll
      for (int i = 0; i < RW; ++i) {
        w[i] = wvec{(WT)0.0f, (WT)0.0f, (WT)0.0f, (WT)0.0f};
        if (k0 + wk < k_end) w[i] = *(const wvec*)(wp[i] + k0);
      }
#pragma unroll
      for (int i = 0; i < RX; ++i) {
        x[i] = xvec{(XT)0.0f, (XT)0.0f, (XT)0.0f, (XT)0.0f};
        if (k0 + xr + XROWS * i < k_end) x[i] = *(const xvec*)(xp[i] + (long long)k0 * p.ldx);
      }
    }
  };
  floatx4 acc[NI][NJ];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  auto put = [&](int k0, int buf) {
    if (k0 + BK > k_end)
#pragma unroll
      for (int i = 0; i < RW; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) w[i][e] = k0 + wk + e < k_end ? w[i][e] : (WT)0.0f;
#pragma unroll
    for (int i = 0; i < RW; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) sW[buf][wk + e][wr + 32 * i] = (float)w[i][e];
#pragma unroll
    for (int i = 0; i < RX; ++i) *(floatx4*)&sX[buf][xr + XROWS * i][xt] = floatx4{(float)x[i][0], (float)x[i][1], (float)x[i][2], (float)x[i][3]};
  };
  // eight steps at a time, the fragments of the next eight read ahead of the products of these
  struct Frag { float a[2][NI], b[2][NJ]; };
  auto read = [&](Frag& f, int buf, int g) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int i = 0; i < NI; ++i) f.a[s][i] = sW[buf][8 * g + 4 * s + kq][wm + 16 * i + l16];
#pragma unroll
      for (int j = 0; j < NJ; ++j) f.b[s][j] = sX[buf][8 * g + 4 * s + kq][wn + 16 * j + l16];
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto multiply = [&](const Frag& f) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(f.b[s][j], f.a[s][i], acc[i][j], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  // Rows of W lie a power of two apart often enough, and then the same columns of all of them in a few of memory's channels: the rows of tiles begin at different
  // places of the contraction and go round it.
  const int n = (k_end - k_first + BK - 1) / BK;
  int k_next = k_first + (int)((long long)(tile % p.tilesM) * n / p.tilesM) * BK;
  const auto next = [&]() {
    const int k = k_next;
    k_next = k + BK < k_end ? k + BK : k_first;
    return k;
  };
  int k1 = next();
  fetch(k1);
  put(k1, 0);
  k1 = next();
  fetch(k1);
  __syncthreads();
  Frag f0, f1;
  read(f0, 0, 0);
  int buf = 0;
#pragma unroll 1
  for (int i = 0; i < n; ++i) {
    read(f1, buf, 1);
    multiply(f0);
    read(f0, buf, 2);
    // the next run of steps goes to the other buffer, and the one behind it is asked for; past the last they are not multiplied
    put(k1, buf ^ 1);
    k1 = next();
    fetch(k1);
    __builtin_amdgcn_sched_barrier(0);
    multiply(f1);
    read(f1, buf, 3);
    multiply(f0);
    __syncthreads();
    read(f0, buf ^ 1, 0);
    multiply(f1);
    buf ^= 1;
  }
  // a lane has four consecutive tokens of a channel
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int m = m0 + wm + 16 * i + l16;
      const long long t = n0 + wn + 16 * j + 4 * kq;
      if (m >= p.M || t >= p.T) continue;
      if (p.splits > 1) *(floatx4*)(p.part + ((long long)split * p.M + m) * p.tp + t) = acc[i][j];
      else finish_quad<YT>(p, acc[i][j], m, t);
    }
}

// Tile shape and parts of the contraction by the time they take.  What 64 steps of the contraction cost (us, on products of 768 .. 8192 channels over 16 .. 5003 tokens): tiles of
// 128 x 128 5.05 alone on a CU, 9.3 two on a CU; of 128 x 64 2.9 and 5.65; of 64 x 64 1.7, 2.85 and 4.2 for one to three; a workgroup's beginning and end as much as one
// more.  Parts cost a launch and their sums' way through the caches.  What the rule weighs, in us: 4096 x 4096 over 200 tokens in tiles of 64 whole 113, in four parts 96, of 128 in
// four 94; over 1024 of 128 whole 331, in two 308, of 64 345; 1000 x 3000 over 700 of 64 whole 82, in four 56; 1013 x 1000 over 5003 of 64 117, of 128 154.
static LinearPlan plan_linear_f32(int M, int K, long long T) {
  const struct { int bm, bn, per; double us[3]; } shapes[3] = {{128, 128, 2, {5.05, 9.3}}, {128, 64, 2, {2.9, 5.65}}, {64, 64, 3, {1.7, 2.85, 4.2}}};
  const int all = (K + 63) / 64;
  LinearPlan best{};
  double least = 0.0;
  for (const auto& s : shapes) {
    const long long n = (long long)((M + s.bm - 1) / s.bm) * ((T + s.bn - 1) / s.bn);
    for (int parts = 1; parts <= 16 && parts <= all; parts *= 2) {
      const int pairs = (all + parts - 1) / parts, used = (all + pairs - 1) / pairs;
      const long long blocks = n * used, round = 256LL * s.per, left = blocks % round;
      if (used > 1 && blocks > round) break;
      const double us = (pairs + 1) * (double(blocks / round) * s.us[s.per - 1] + (left ? s.us[(left + 255) / 256 - 1] : 0.0)) +
                        (used > 1 ? 2.5 + 1.2e-6 * used * (double)M * (double)T : 0.0);
      if (least > 0.0 && us >= least) continue;
      least = us;
      best = LinearPlan{0, s.bm, s.bn, used, pairs, used > 1 ? (size_t)used * M * ((T + 7) / 8 * 8) * 4 : 0};
    }
  }
  return best;
}
static LinearPlan plan_linear(int M, int K, long long T, int w_dtype, int x_dtype) {
  return w_dtype == STRP_BF16 && x_dtype == STRP_BF16 ? plan_linear_bf16(M, K, T) : plan_linear_f32(M, K, T);
}

template <typename WT, typename XT, typename YT>
static void launch_f32(strp_ctx* ctx, const LinearP& p, const LinearPlan& plan) {
  const dim3 grid((unsigned)((long long)p.tilesM * p.tilesN * p.splits)), block(256);
  if (plan.bn == 128) hipLaunchKernelGGL((linear_f32_kernel<128, 128, WT, XT, YT>), grid, block, 0, ctx->stream, p);
  else if (plan.bm == 128) hipLaunchKernelGGL((linear_f32_kernel<128, 64, WT, XT, YT>), grid, block, 0, ctx->stream, p);
  else hipLaunchKernelGGL((linear_f32_kernel<64, 64, WT, XT, YT>), grid, block, 0, ctx->stream, p);
}
template <typename WT, typename XT>
static void launch_linear_f32(strp_ctx* ctx, LinearP p, const LinearPlan& plan, int y_dtype) {
  p.tilesM = (p.M + plan.bm - 1) / plan.bm;
  p.tilesN = (int)((p.T + plan.bn - 1) / plan.bn);
  p.splits = plan.splits;
  p.pairs = plan.pairs;
  p.tp = (p.T + 7) / 8 * 8;
  if (y_dtype == STRP_BF16) launch_f32<WT, XT, __bf16>(ctx, p, plan);
  else launch_f32<WT, XT, float>(ctx, p, plan);
  if (p.splits > 1) launch_linear_join(ctx, p, y_dtype);
}

}  // namespace strp

using namespace strp;

extern "C" {

size_t strp_linear_workspace_bytes(int32_t M, int32_t K, int64_t T, strp_dtype w_dtype, strp_dtype x_dtype) {
  if (M <= 0 || K <= 0 || T <= 0 || M > (1 << 30) || K > (1 << 30)) return 0;
  const size_t part = plan_linear(M, K, T, w_dtype, x_dtype).part_bytes;
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
  if (in->M > (1 << 30) || in->K > (1 << 30) || in->T > 1LL << 31) return fail(ctx, STRP_EINVAL, "linear: M or K above 2^30, or T above 2^31");
  LinearP p{in->W, in->X, in->bias, in->R, in->Y, in->M, in->K, in->act, in->T, in->ldw, in->ldx, in->ldr, in->ldy};
  p.splits = 1;
  const LinearPlan plan = plan_linear(p.M, p.K, p.T, in->w_dtype, in->x_dtype);
  if ((long long)((p.M + plan.bm - 1) / plan.bm) * ((p.T + plan.bn - 1) / plan.bn) > MAX_TILES) return fail(ctx, STRP_EINVAL, "linear: more tiles than a launch holds");
  if (plan.part_bytes) {
    if (!ctx->ws) return fail(ctx, STRP_ENOMEM, "linear: no workspace set");
    Arena arena(ctx);
    STRP_TAKE(ctx, arena, part, float, plan.part_bytes / 4);
    p.part = part;
  }
  OnDevice on(ctx);
  if (!on.ok()) return fail(ctx, STRP_EHIP, "linear: device %d cannot be made current", ctx->device);
  const double M = in->M, K = in->K, T = (double)in->T;
  ProfScope ps(ctx, "linear", 2.0 * M * K * T, bytes_of(in->w_dtype) * M * K + bytes_of(in->x_dtype) * K * T + bytes_of(in->y_dtype) * M * T * (in->R ? 2 : 1));
  const bool wb = in->w_dtype == STRP_BF16, xb = in->x_dtype == STRP_BF16;
  if (wb && xb) launch_linear_bf16(ctx, p, plan, in->y_dtype);
  else if (wb) launch_linear_f32<__bf16, float>(ctx, p, plan, in->y_dtype);
  else if (xb) launch_linear_f32<float, __bf16>(ctx, p, plan, in->y_dtype);
  else launch_linear_f32<float, float>(ctx, p, plan, in->y_dtype);
  STRP_HIP(ctx, hipGetLastError());
  return STRP_OK;
}

}  // extern "C"
