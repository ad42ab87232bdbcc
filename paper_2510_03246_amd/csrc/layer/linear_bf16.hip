// act(W X + bias) + R with W and X in bf16: v_mfma_f32_16x16x32_bf16, fp32 sums.
//
// W has its contraction contiguous, X its tokens, so a fragment of W is 16 bytes of a row and a fragment of X is a column: it is
// read from LDS by ds_read_b64_tr_b16, which hands the 16 lanes of a group the 16 columns of four rows.  The accumulator is that of
// (tokens x channels): a lane has four consecutive tokens of one channel.
#include "linear.h"

#include <algorithm>

namespace strp {

// Which tile a workgroup has: workgroups go to the eight XCDs in turn, and the per that an XCD holds at a time are neighbours, eight
// tiles of channels by per / 8 of tokens, so that its L2 serves them from 8 + per / 8 panels.
__device__ __forceinline__ void tile_of(int b, int blocks, int per, int tilesM, int tilesN, int& tm, int& tn) {
  const int round = 8 * per, full = blocks / round * round;
  int q;
  if (b < full) {
    q = b / round * round + (b & 7) * per + b % round / 8;
  } else {
    const int x = b & 7, rem = blocks - full;
    q = full + x * (rem >> 3) + min(x, rem & 7) + ((b - full) >> 3);
  }
  const int band = q / (8 * tilesN), r = q - band * 8 * tilesN, h = min(8, tilesM - 8 * band);
  tn = r / h;
  tm = 8 * band + r - tn * h;
}

// X of 32 steps lies in LDS as 32 rows of BN tokens, in blocks of 16 tokens whose order depends on the row so that the rows that a read
// touches at once are in different banks.
template <int BN>
__device__ __forceinline__ constexpr int block_turn(int k) {
  return BN >= 128 ? ((k & 3) | ((k >> 1) & 4)) : (((k >> 1) & 1) | ((k >> 2) & 2));
}

// What becomes of a wavefront's sums: acc[i][j] has tokens 16 j + 4 (lane / 16) .. + 3 of channel m + 16 i, tokens from t on.  bf16: four lanes
// exchange their quads so that each has two runs of eight tokens, and every row is written in 64 contiguous bytes an instruction.
template <typename YT, int NI>
__device__ __forceinline__ void finish_tile(const LinearP& p, const floatx4 (&acc)[NI][4], int m, long long t, YT* out, long long ldo, const float* bias,
                                            const YT* res, int act) {
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int mi = m + 16 * i;
    const bool row = mi < p.M;
    const int mc = row ? mi : p.M - 1;
    const float b = bias ? bias[mc] : 0.0f;
    const YT* R = res ? res + (long long)mc * p.ldr : nullptr;
    YT* Y = out + (long long)mc * ldo;
    if constexpr (sizeof(YT) == 4) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const long long tj = t + 16 * j + 4 * g;
        floatx4 v = acc[i][j], r = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        const bool ok = row && tj < p.T;
        if (R && ok) r = *(const floatx4*)(R + tj);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = activate(v[e] + b, act) + r[e];
        if (!ok) continue;
        if (tj + 4 <= p.T) *(floatx4*)(Y + tj) = v;
        else
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (tj + e < p.T) Y[tj + e] = v[e];
      }
    } else {
      floatx4 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[j][e] = activate(acc[i][j][e] + b, act);
      // slots (j1 j0) x lanes (g1 g0) of quads 8 j1 + 4 j0 + 2 g1 + g0  ->  lanes (j0 g1), slots (j1 g0); in fp32 where the residual is to be added before
      // the one rounding, else in bf16
      const auto swap32 = [](unsigned& a, unsigned& b2) { const auto s = __builtin_amdgcn_permlane32_swap(a, b2, false, false); a = s[0]; b2 = s[1]; };
      const auto swap16 = [](unsigned& a, unsigned& b2) { const auto s = __builtin_amdgcn_permlane16_swap(a, b2, false, false); a = s[0]; b2 = s[1]; };
      if (R) {
        const auto turn = [&](int j1) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float v0 = v[2 * j1][e], v1 = v[2 * j1 + 1][e];       // not bit_cast of an element of a vector: that takes the first
            unsigned a = __builtin_bit_cast(unsigned, v0), c = __builtin_bit_cast(unsigned, v1);
            swap32(a, c);
            swap16(a, c);
            v[2 * j1][e] = __builtin_bit_cast(float, a);
            v[2 * j1 + 1][e] = __builtin_bit_cast(float, c);
          }
        };
        turn(0);
        turn(1);
      }
#pragma unroll
      for (int j1 = 0; j1 < 2; ++j1) {
        const long long tj = t + 32 * j1 + 8 * g;
        const bool ok = row && tj < p.T;
        uint4 out;
        if (R) {
          bf16x8 r;
          if (ok) r = *(const bf16x8*)(R + tj);
          bf16x8 y;
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = (__bf16)(v[2 * j1 + (e >> 2)][e & 3] + (ok ? (float)r[e] : 0.0f));
          out = __builtin_bit_cast(uint4, y);
        } else {
          unsigned q[4];
#pragma unroll
          for (int j0 = 0; j0 < 2; ++j0)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              q[2 * j0 + e] = __builtin_bit_cast(unsigned, bf16x2{(__bf16)v[2 * j1 + j0][2 * e], (__bf16)v[2 * j1 + j0][2 * e + 1]});
          swap32(q[0], q[2]);
          swap32(q[1], q[3]);
          swap16(q[0], q[2]);
          swap16(q[1], q[3]);
          out = make_uint4(q[0], q[1], q[2], q[3]);
        }
        if (!ok) continue;
        if (tj + 8 <= p.T) *(uint4*)(Y + tj) = out;
        else {
          const bf16x8 y = __builtin_bit_cast(bf16x8, out);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (tj + e < p.T) Y[tj + e] = y[e];
        }
      }
    }
  }
}

// Tiles of (WM 16 NI) channels x (64 WN) tokens, a wavefront 16 NI x 64, in steps of 32 of the contraction.  W comes in pairs of steps, 128 bytes of a row: the
// line that memory hands out whole.  LDS holds three pairs of W and four steps of X, and all but what is being multiplied is on its way.  A remainder of the
// contraction is the first pair and goes through registers, zeros from K on.  What bounds it is a step's matrix instructions and reads of LDS, which overlap in part (64 steps of
// a tile of 256 1.8 us, the matrix instructions alone 0.85; the matrix cores are busy 42 % of the time), in the largest products also power: 8192 x 2048 over 2048 tokens
// 62 us, 1.1 PFLOP/s; 4096 x 4915 over 32768 1.19 to 1.27 ms, 1.04 to 1.11; 768 x 768 over 2048 11.8 us.
template <int WM, int WN, int NI, typename YT>
__global__ __launch_bounds__(64 * WM * WN, WM * WN >= 8 ? 1 : 2) void linear_tile_kernel(const LinearP p) {
  constexpr int NW = WM * WN, BM = WM * 16 * NI, BN = WN * 64, PAIR = BM * 128, STEP = BN * 64, XAT = 3 * PAIR, RPI = 512 / BN;     // RPI: rows of X in a KB
  constexpr int LW = BM / 8 / NW, LX = BN / 16 / NW;      // loads of a pair, of a step
  static_assert(BM % (8 * NW) == 0 && BN % (16 * NW) == 0, "whole pieces for every wavefront");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[3 * PAIR + 4 * STEP];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
  const int tiles = p.tilesM * p.tilesN, split = (int)blockIdx.x / tiles;
  int tm, tn;
  tile_of((int)blockIdx.x - split * tiles, tiles, NW >= 8 ? 32 : 64, p.tilesM, p.tilesN, tm, tn);
  const int m0 = tm * BM;
  const long long n0 = (long long)tn * BN;
  const __bf16* W = (const __bf16*)p.W;
  const __bf16* X = (const __bf16*)p.X;
  const int all = (p.K + 63) / 64, p0 = split * p.pairs, p1 = min(all, p0 + p.pairs);
  const int rest = p1 == all ? p.K & 63 : 0;               // this part has the remainder
  const int whole = p1 - p0 - (rest ? 1 : 0), n = 2 * (p1 - p0), first = rest ? 1 : 0;

  // this wavefront's KBs: eight rows of W (eight chunks of 16 bytes each, in an order that depends on the row), RPI rows of X
  const __bf16* srcW[LW];
  const __bf16* srcX[LX];
  int chunkW[LW], rowX[LX];
  const long long t_last = (p.T - 1) / 8 * 8;
  const unsigned base = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem;
#pragma unroll
  for (int i = 0; i < LW; ++i) {
    const int r = 8 * (wave + NW * i) + (lane >> 3);
    chunkW[i] = 8 * ((lane & 7) ^ ((r >> 1) & 7));
    srcW[i] = W + (long long)min(m0 + r, p.M - 1) * p.ldw + chunkW[i];
  }
#pragma unroll
  for (int i = 0; i < LX; ++i) {
    const int c = lane % (64 / RPI);
    rowX[i] = (wave + NW * i) * RPI + lane / (64 / RPI);
    const long long t = n0 + 16 * ((c >> 1) ^ block_turn<BN>(rowX[i])) + 8 * (c & 1);
    srcX[i] = X + (t < p.T ? t : t_last) + (long long)rowX[i] * p.ldx;
  }
  // pairs and steps past the last re-read it and are never multiplied
  auto issue_w = [&](int pr) {
    if (whole == 0) return;
    const long long k = (long long)(p0 + min(pr - first, whole - 1)) * 64;
#pragma unroll
    for (int i = 0; i < LW; ++i) copy_to_lds(srcW[i] + k, base + (unsigned)(pr % 3) * PAIR + (unsigned)(wave + NW * i) * 1024);
  };
  auto issue_x = [&](int s) {
    if (whole == 0) return;
    const long long k = (long long)p0 * 64 + 32 * min(s - 2 * first, 2 * whole - 1);
#pragma unroll
    for (int i = 0; i < LX; ++i) copy_to_lds(srcX[i] + k * p.ldx, base + XAT + (unsigned)(s & 3) * STEP + (unsigned)(wave + NW * i) * 1024);
  };
  if (rest) {
    const int k0 = p.K - rest;
#pragma unroll
    for (int i = 0; i < LW; ++i) {
      const int k = k0 + chunkW[i];
      bf16x8 v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (__bf16)0.0f;
      if (k < p.K) {
        v = *(const bf16x8*)(srcW[i] + k0);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = k + e < p.K ? v[e] : (__bf16)0.0f;
      }
      *(bf16x8*)(smem + (wave + NW * i) * 1024 + 16 * lane) = v;
    }
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < LX; ++i) {
        uintx4 v = uintx4{0u, 0u, 0u, 0u};
        if (k0 + 32 * s + rowX[i] < p.K) v = *(const uintx4*)(srcX[i] + (long long)(k0 + 32 * s) * p.ldx);
        *(uintx4*)(smem + XAT + s * STEP + (wave + NW * i) * 1024 + 16 * lane) = v;
      }
  } else {
    issue_x(0);
    issue_w(0);
    issue_x(1);
  }
  issue_x(2);
  issue_w(1);
  issue_x(3);

  floatx4 acc[NI][4];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  const int kg = lane >> 4, l16 = lane & 15;
  const unsigned offW = base + (unsigned)((wm * NI * 16 + l16) * 128 + ((kg ^ (l16 >> 1)) * 16));
  unsigned offX[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int k = 8 * kg + (l16 >> 2);
    offX[j] = base + XAT + (unsigned)(k * (BN * 2) + ((wn * 4 + j) ^ block_turn<BN>(k)) * 32 + (l16 & 3) * 8);
  }
  struct XF { short4v lo[4], hi[4]; };
  auto read_x = [&](XF& f, int s, int j0, int j1) {
    const unsigned at = (unsigned)(s & 3) * STEP;
#pragma unroll
    for (int j = j0; j < j1; ++j) {
      f.lo[j] = read_turned(offX[j] + at);
      f.hi[j] = read_turned(offX[j] + at + 4 * (BN * 2));
    }
  };
  unsigned pair_at = 0;                                    // where the pair of the step being read lies
  auto read_w = [&](bf16x8& f, int odd, int i) {
    f = *(const __attribute__((address_space(3))) bf16x8*)(size_t)((offW ^ (unsigned)(64 * odd)) + pair_at + i * 2048);
  };
  auto row = [&](floatx4 (&c)[4], const bf16x8& w, const XF& x) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      c[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, __builtin_shufflevector(x.lo[j], x.hi[j], 0, 1, 2, 3, 4, 5, 6, 7)), w, c[j], 0, 0, 0);
  };
  bf16x8 wa, wb;
  // A step.  Its fragments of X are in registers as it begins, and so is its first one of W.  Halfway through, the wavefronts meet: the next step has landed, and
  // nobody reads this step's X or the pair before this step's any more, so their places are asked for again; the second half reads the next step's fragments.
  auto step = [&](int s, int odd, const XF& xc, XF& xn) {
    constexpr int HALF = NI / 2;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      if (i + 1 < NI) read_w(i & 1 ? wa : wb, odd, i + 1);
      if (i >= HALF) read_x(xn, s + 1, (i - HALF) * 4 / HALF, (i - HALF + 1) * 4 / HALF);      // past the last step: a slot that is never multiplied
      if (i + 1 == NI) {
        if (odd) pair_at = pair_at == 2 * PAIR ? 0 : pair_at + PAIR;
        read_w(wa, !odd, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
      row(acc[i], i & 1 ? wb : wa, xc);
      __builtin_amdgcn_sched_barrier(0);
      if (i + 1 == HALF) {
        wait_loads<2 * LX + LW>();
        __builtin_amdgcn_s_barrier();
        issue_x(s + 4);
        if (!odd) issue_w((s >> 1) + 2);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  XF x0, x1;
  wait_loads_and_lds<LW + 3 * LX>();
  __syncthreads();
  read_x(x0, 0, 0, 4);
  read_w(wa, 0, 0);
#pragma unroll 1
  for (int s = 0; s < n; s += 2) {
    step(s, 0, x0, x1);
    step(s + 1, 1, x1, x0);
  }
  wait_loads<0>();
  const int m = m0 + wm * NI * 16 + l16;
  const long long t = n0 + wn * 64;
  if (p.splits > 1) finish_tile<float, NI>(p, acc, m, t, p.part + (long long)split * p.M * p.tp, p.tp, nullptr, nullptr, STRP_ACT_NONE);
  else finish_tile<YT, NI>(p, acc, m, t, (YT*)p.Y, p.ldy, p.bias, (const YT*)p.R, p.act);
}

// Few tokens (T <= 16 NT): W is the traffic, read once straight into fragments (a lane has 16 bytes of a row), the contraction in parts among the NW wavefronts
// of a workgroup, which add their sums up in LDS.  X goes to LDS as it lies, a run of rows at a time, and is read turned.  A workgroup has 16 channels.
// What bounds it is the rate of its reads, each of 16 rows: 2.6 TB/s of W with a workgroup to a CU and 3.0 from two on (4096 x 4096 one token 13.2 us, 8192 x 2048 11.4; with W in the last-level cache 11.9, 10.2); below
// that a launch and the latencies of X, W and the sums (768 x 768 4.1 us).  Asking for X two runs ahead, beginning at different places of the contraction, both
// steps of a line to one wavefront and 32 channels a workgroup changed it by less than 10 % either way.
constexpr int FEW_WAVES = 8;
template <int NT, typename YT>
__global__ __launch_bounds__(64 * FEW_WAVES, 2) void linear_few_kernel(const LinearP p) {
  constexpr int NW = FEW_WAVES, ROW = 32 * NT;             // bytes of a row of X in LDS: 16 NT tokens
  constexpr int PER = NT == 1 ? 4 : 2, KC = 32 * NW * PER, XC = KC * 2 * NT / (64 * NW);      // steps of a wavefront in a run, rows of X in it, chunks of X a thread moves
  static_assert(NW * NT * 1024 <= 2 * KC * ROW, "the sums lie where X was");
  __shared__ __attribute__((aligned(16))) unsigned char sX[2][KC * ROW];
  floatx4(*sums)[NT][64] = (floatx4(*)[NT][64])&sX[0][0];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), kg = lane >> 4, l16 = lane & 15;
  const int m0 = (int)blockIdx.x * 16;
  const __bf16* X = (const __bf16*)p.X;
  const __bf16* W = (const __bf16*)p.W + (long long)min(m0 + l16, p.M - 1) * p.ldw;
  floatx4 acc[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) acc[t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  const unsigned base = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)sX;
  const int t_last = (int)((p.T - 1) / 8);                 // last chunk of eight tokens
  const uintx4 zero = uintx4{0u, 0u, 0u, 0u};
  // a wavefront's steps of a run are k0 + 32 (wave + NW j); what lies behind K is zero
  struct Run { uintx4 w[PER]; };
  auto ask_w = [&](Run& r, int k0) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int k = k0 + 32 * (wave + NW * j) + 8 * kg;
      r.w[j] = k < p.K ? *(const uintx4*)(W + k) : zero;
    }
  };
  uintx4 x[XC];
  auto ask_x = [&](int k0) {
#pragma unroll
    for (int c = 0; c < XC; ++c) {
      const int at = tid + 64 * NW * c, k = k0 + at / (2 * NT), ch = at % (2 * NT);
      x[c] = k < p.K && ch <= t_last ? *(const uintx4*)(X + (long long)k * p.ldx + 8 * ch) : zero;
    }
  };
  auto put_x = [&](int buf) {
#pragma unroll
    for (int c = 0; c < XC; ++c) *(uintx4*)(sX[buf] + (tid + 64 * NW * c) * 16) = x[c];
  };
  auto multiply = [&](const Run& r, int k0, int buf) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int kl = 32 * (wave + NW * j);
      if (k0 + kl >= p.K) break;
      bf16x8 w = __builtin_bit_cast(bf16x8, r.w[j]);
      if (k0 + kl + 32 > p.K)
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = k0 + kl + 8 * kg + e < p.K ? w[e] : (__bf16)0.0f;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const unsigned at = base + (unsigned)(buf * KC * ROW + (kl + 8 * kg + (l16 >> 2)) * ROW + 32 * t + (l16 & 3) * 8);
        const bf16x8 xf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(read_turned(at), read_turned(at + 4 * ROW), 0, 1, 2, 3, 4, 5, 6, 7));
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf, w, acc[t], 0, 0, 0);
      }
    }
  };
  // W is asked for two runs ahead, X one
  Run ra, rb;
  ask_x(0);
  ask_w(ra, 0);
  ask_w(rb, KC);
  put_x(0);
  __syncthreads();
#pragma unroll 1
  for (int k0 = 0; k0 < p.K; k0 += 2 * KC) {
    ask_x(k0 + KC);
    multiply(ra, k0, 0);
    ask_w(ra, k0 + 2 * KC);
    put_x(1);
    __syncthreads();
    if (k0 + KC >= p.K) break;
    ask_x(k0 + 2 * KC);
    multiply(rb, k0 + KC, 1);
    ask_w(rb, k0 + 3 * KC);
    put_x(0);
    __syncthreads();
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) sums[wave][t][lane] = acc[t];
  __syncthreads();
  // four tokens of a channel to a thread, the wavefronts' sums in their order
  if (tid >= NT * 64) return;
  const int t = wave, m = m0 + l16, tok = 16 * t + 4 * kg;
  floatx4 v = sums[0][t][lane];
#pragma unroll
  for (int s = 1; s < NW; ++s) v += sums[s][t][lane];
  if (m < p.M && tok < p.T) finish_quad<YT>(p, v, m, tok);
}

// Sums of the parts in their order: a thread has four tokens of a channel.
template <typename YT>
__global__ __launch_bounds__(256) void linear_join_kernel(const LinearP p) {
  const long long quads = p.tp / 4, i = (long long)blockIdx.x * 256 + threadIdx.x;
  const int m = (int)(i / quads);
  const long long t = (i - m * quads) * 4;
  if (m >= p.M || t >= p.T) return;
  floatx4 v = *(const floatx4*)(p.part + (long long)m * p.tp + t);
  for (int s = 1; s < p.splits; ++s) v += *(const floatx4*)(p.part + ((long long)s * p.M + m) * p.tp + t);
  finish_quad<YT>(p, v, m, t);
}

void launch_linear_join(strp_ctx* ctx, const LinearP& p, int y_dtype) {
  const dim3 grid((unsigned)((p.M * (p.tp / 4) + 255) / 256)), block(256);
  if (y_dtype == STRP_BF16) hipLaunchKernelGGL((linear_join_kernel<__bf16>), grid, block, 0, ctx->stream, p);
  else hipLaunchKernelGGL((linear_join_kernel<float>), grid, block, 0, ctx->stream, p);
}

// Tile shape and parts of the contraction by the time they take.  A workgroup's pair of steps takes the longer the more workgroups share its CU (us, measured on
// products of 768 .. 8192 channels over 128 .. 8192 tokens): tiles of 256 1.8, alone on a CU; of 128 0.65 alone, 1.25 two on a CU; of 64 0.42, 0.6, 0.75 and 0.9 for
// one to four.  Parts cost a launch and their sums' way through memory.  What the rule weighs, in us: 8192 x 2048 over 1024 tokens in tiles of 256 57, of 128 41, over 2048
// 65 against 80; 768 x 768 over 2048 in tiles of 128 13.5, of 64 11.7; 4096 x 4096 over 128 in tiles of 64 whole 30, in two parts 20, in four 17.5.
// Few tokens: a workgroup of 16 channels goes through the whole contraction by itself, which the tiles' parts overtake where it is long or there are many workgroups to a CU.
// One token, us, few against tiles: 768 x 768 4.1, 6.9; 4096 x 4096 13.9, 15.9; 16384 x 1000 12.1, 12.9; 2048 x 8192 21.7, 16.2; 50000 x 768 24, 17.5.  32 tokens: 2048 x 2048
// 7.5, 9.4; 4096 x 4096 16.3, 13.4; 8192 x 2048 14.0, 12.2.  33 tokens and more (with twice the channels): 2048 x 2048 12.0, 10.0; 4096 x 4096 22.6, 13.8.
LinearPlan plan_linear_bf16(int M, int K, long long T) {
  LinearPlan best{LINEAR_FEW, 16, 32, 1, 0, 0};
  if (T <= 32 && (long long)K * std::max(M, 4096) <= 1 << (T <= 16 ? 24 : 23)) return best;
  const struct { int kind, b, per; double us[4]; } shapes[3] = {
      {LINEAR_TILE_LARGE, 256, 1, {1.8}}, {LINEAR_TILE, 128, 2, {0.65, 1.25}}, {LINEAR_TILE_SMALL, 64, 4, {0.42, 0.6, 0.75, 0.9}}};
  const int all = (K + 63) / 64;
  double least = 0.0;
  for (const auto& s : shapes) {
    const long long n = ((M + s.b - 1) / s.b) * ((T + s.b - 1) / s.b);
    for (int parts = 1; parts <= 16 && parts <= all; parts *= 2) {
      const int pairs = (all + parts - 1) / parts, used = (all + pairs - 1) / pairs;
      const long long blocks = n * used, round = 256LL * s.per, left = blocks % round;
      if (used > 1 && blocks > round) break;
      const double us = pairs * (double(blocks / round) * s.us[s.per - 1] + (left ? s.us[(left + 255) / 256 - 1] : 0.0)) +
                        (used > 1 ? 1.5 + 8e-6 / 4.5 * used * (double)M * (double)T : 0.0);
      if (least > 0.0 && us >= least) continue;
      least = us;
      best = LinearPlan{s.kind, s.b, s.b, used, pairs, used > 1 ? (size_t)used * M * ((T + 7) / 8 * 8) * 4 : 0};
    }
  }
  return best;
}

template <typename YT>
static void launch_tiles(strp_ctx* ctx, const LinearP& p, const LinearPlan& plan) {
  const dim3 grid((unsigned)((long long)p.tilesM * p.tilesN * p.splits));
  if (plan.kind == LINEAR_TILE_LARGE) hipLaunchKernelGGL((linear_tile_kernel<2, 4, 8, YT>), grid, dim3(512), 0, ctx->stream, p);
  else if (plan.kind == LINEAR_TILE) hipLaunchKernelGGL((linear_tile_kernel<2, 2, 4, YT>), grid, dim3(256), 0, ctx->stream, p);
  else hipLaunchKernelGGL((linear_tile_kernel<2, 1, 2, YT>), grid, dim3(128), 0, ctx->stream, p);
}

template <typename YT>
static void launch_few(strp_ctx* ctx, const LinearP& p) {
  const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(p.tilesM), dim3(64 * FEW_WAVES), 0, ctx->stream, p); };
  if (p.T <= 16) go(linear_few_kernel<1, YT>);
  else go(linear_few_kernel<2, YT>);
}

void launch_linear_bf16(strp_ctx* ctx, LinearP p, const LinearPlan& plan, int y_dtype) {
  p.tilesM = (p.M + plan.bm - 1) / plan.bm;
  if (plan.kind == LINEAR_FEW) {
    if (y_dtype == STRP_BF16) launch_few<__bf16>(ctx, p);
    else launch_few<float>(ctx, p);
    return;
  }
  p.tilesN = (int)((p.T + plan.bn - 1) / plan.bn);
  p.splits = plan.splits;
  p.pairs = plan.pairs;
  p.tp = (p.T + 7) / 8 * 8;
  if (y_dtype == STRP_BF16) launch_tiles<__bf16>(ctx, p, plan);
  else launch_tiles<float>(ctx, p, plan);
  if (p.splits > 1) launch_linear_join(ctx, p, y_dtype);
}

}  // namespace strp
