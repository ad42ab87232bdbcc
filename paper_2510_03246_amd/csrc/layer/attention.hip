// Causal attention over whole prompts, heads in groups, sequences packed along the tokens.
//
//   c_t = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q_t . k_j - m),  j from the start of t's sequence to t,
// in one pass over the keys with the running maximum m and sum of the softmax.  A workgroup has the queries of one head at
// consecutive tokens and walks the keys from the start of its first query's sequence; every query has a range [lo, t] of
// keys, so that a tile of queries that crosses from one sequence into the next needs nothing of its own.
#include "layer_ops.h"

#include <cmath>

namespace strp {

struct AttnP {
  const void* Q;
  const void* K;
  const void* V;
  void* C;
  const int32_t* seq_start;
  const int32_t* kv_of_head;
  int heads, kv_heads, group, dh, n_seq, tiles;
  long long T, ldq, ldk, ldv, ldc;
  float scale_log2e;
};

// First key of token t's sequence; t + 1 where t is in none.
__device__ __forceinline__ int first_key(const AttnP& p, int t) {
  if (t >= p.T) return t + 1;
  if (!p.seq_start) return 0;
  int a = -1, b = p.n_seq + 1;             // seq_start[a] <= t < seq_start[b]
  while (b - a > 1) {
    const int c = (a + b) >> 1;
    if (p.seq_start[c] <= t) a = c;
    else b = c;
  }
  if (a < 0 || a == p.n_seq) return t + 1;
  const int s = p.seq_start[a];
  return s < 0 ? 0 : s;
}

__device__ __forceinline__ int kv_head_of(const AttnP& p, int head) {
  if (!p.kv_of_head) return head / p.group;
  const int g = p.kv_of_head[head];
  return g < 0 ? 0 : (g < p.kv_heads ? g : p.kv_heads - 1);
}

// What a value that is not finite adds to a sum of products with ones and zeros: 1 for +inf, 64 for -inf, 4096 for NaN.  Sums over up to 63
// keys keep the three counts apart, and all of it is exact in bf16 and fp32.
__device__ __forceinline__ float not_finite_mark(float v) {
  return v != v ? 4096.0f : (v == INFINITY ? 1.0f : (v == -INFINITY ? 64.0f : 0.0f));
}
__device__ __forceinline__ float of_marks(float n) {
  if (n == 0.0f) return 0.0f;
  if (n < 64.0f) return INFINITY;
  const int c = (int)n;
  return c < 4096 && (c & 63) == 0 ? -INFINITY : NAN;
}

// Products of fp32 (v_mfma_f32_32x32x2_f32).  Four wavefronts of 32 queries, keys 64 at a time.  S = K^T Q has a query to a lane (the keys of
// its 16 registers are 8 (e / 4) + 4 (lane / 32) + e % 4), so the softmax needs one exchange between the lane's two halves, and
// the registers of P are the second operand of V P as they are.
template <typename E, int DHP>
__global__ __launch_bounds__(256, 2) void attention_f32_kernel(const AttnP p) {
  constexpr int KT = 64, PITCH = KT + 4, NC = DHP / 32, CHUNKS = KT / 4;
  __shared__ __attribute__((aligned(16))) float sK[DHP][PITCH], sV[DHP][PITCH];
  __shared__ int lows[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = lane >> 5, l32 = lane & 31;
  const int head = blockIdx.y, tile = p.tiles - 1 - (int)blockIdx.x;       // the tiles with most keys first
  const int q0 = tile * 128, q = q0 + wave * 32 + l32;
  const int lo = first_key(p, q);
  const bool some = lo <= q;
  const int kv = kv_head_of(p, head);
  const E* Kh = (const E*)p.K + (long long)kv * p.dh * p.ldk;
  const E* Vh = (const E*)p.V + (long long)kv * p.dh * p.ldv;

  int wlo = some ? lo : 0x7fffffff;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) wlo = min(wlo, __shfl_xor(wlo, o, 64));
  if (lane == 0) lows[wave] = wlo;
  float qf[DHP / 2];
#pragma unroll
  for (int s = 0; s < DHP / 2; ++s) qf[s] = some && 2 * s + h < p.dh ? (float)((const E*)p.Q)[((long long)head * p.dh + 2 * s + h) * p.ldq + q] : 0.0f;
  for (int i = tid; i < (DHP - p.dh) * KT; i += 256) sK[p.dh + i / KT][i % KT] = sV[p.dh + i / KT][i % KT] = 0.0f;
  __syncthreads();
  const int low = min(min(lows[0], lows[1]), min(lows[2], lows[3]));
  if (low == 0x7fffffff) return;                 // no query of this tile is in a sequence
  const int last = q0 + 127 < (int)(p.T - 1) ? q0 + 127 : (int)(p.T - 1);

  floatx16 O[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) O[c][e] = 0.0f;
  float m = -INFINITY, l = 0.0f;
  for (int k0 = low & ~(KT - 1); k0 <= last; k0 += KT) {
    __syncthreads();
#pragma unroll 2
    for (int i = tid; i < p.dh * CHUNKS; i += 256) {
      const int r = i / CHUNKS, c = (i % CHUNKS) * 4;
      float k[4] = {0.0f, 0.0f, 0.0f, 0.0f}, v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      if (k0 + c < p.T) {
        load_floats<4>(Kh + (long long)r * p.ldk + k0 + c, k);
        load_floats<4>(Vh + (long long)r * p.ldv + k0 + c, v);
      }
      *(floatx4*)&sK[r][c] = floatx4{k[0], k[1], k[2], k[3]};
      *(floatx4*)&sV[r][c] = floatx4{v[0], v[1], v[2], v[3]};
    }
    __syncthreads();
    if (!__any(some && q >= k0 && lo < k0 + KT)) continue;               // nothing here that this wavefront sees
    const bool whole = __all(some && lo <= k0 && q >= k0 + KT - 1);
    floatx16 S[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) S[u][e] = 0.0f;
#pragma unroll
    for (int s = 0; s < DHP / 2; ++s)
#pragma unroll
      for (int u = 0; u < 2; ++u) S[u] = __builtin_amdgcn_mfma_f32_32x32x2f32(sK[2 * s + h][32 * u + l32], qf[s], S[u], 0, 0, 0);
    float mt = -INFINITY;
    if (!whole) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int key = k0 + 32 * u + 8 * (e >> 2) + 4 * h + (e & 3);
          if (key < lo || key > q) S[u][e] = -INFINITY;
        }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) mt = __builtin_elementwise_maximum(mt, S[u][e]);
    mt = __builtin_elementwise_maximum(mt, __shfl_xor(mt, 32, 64));
    const float mn = __builtin_elementwise_maximum(m, mt), ref = mn == -INFINITY ? 0.0f : mn * p.scale_log2e;
    const float fac = __builtin_amdgcn_exp2f(m * p.scale_log2e - ref);
    m = mn;
    float sum = 0.0f;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        S[u][e] = __builtin_amdgcn_exp2f(S[u][e] * p.scale_log2e - ref);
        sum += S[u][e];
      }
    l = l * fac + sum;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) O[c][e] *= fac;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      bool odd = false;                  // a value that is not finite, where some key is not seen by every query
      if (!whole)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const floatx4 v = *(const floatx4*)&sV[32 * c + l32][32 * u + 8 * g + 4 * h];
#pragma unroll
            for (int e = 0; e < 4; ++e) odd |= !(fabsf(v[e]) < INFINITY);
          }
      if (__any(odd)) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          floatx16 marks;
#pragma unroll
          for (int e = 0; e < 16; ++e) marks[e] = 0.0f;
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int at = 32 * u + 8 * (e >> 2) + 4 * h + (e & 3), key = k0 + at;
            const float v = sV[32 * c + l32][at], mark = not_finite_mark(v);
            marks = __builtin_amdgcn_mfma_f32_32x32x2f32(mark, key >= lo && key <= q ? 1.0f : 0.0f, marks, 0, 0, 0);
            O[c] = __builtin_amdgcn_mfma_f32_32x32x2f32(mark != 0.0f ? 0.0f : v, S[u][e], O[c], 0, 0, 0);
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) O[c][e] += of_marks(marks[e]);
        }
      } else {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const floatx4 v = *(const floatx4*)&sV[32 * c + l32][32 * u + 8 * g + 4 * h];
#pragma unroll
            for (int e = 0; e < 4; ++e) O[c] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[e], S[u][4 * g + e], O[c], 0, 0, 0);
          }
      }
    }
  }
  l += __shfl_xor(l, 32, 64);
  const float inv = 1.0f / l;
  if (!some) return;
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int r = 32 * c + 8 * (e >> 2) + 4 * h + (e & 3);
      if (r < p.dh) ((E*)p.C)[((long long)head * p.dh + r) * p.ldc + q] = (E)(O[c][e] * inv);
    }
}

template <typename E>
static void launch_attention_f32(strp_ctx* ctx, const AttnP& p) {
  const dim3 grid(p.tiles, p.heads), block(256);
  if (p.dh <= 64) hipLaunchKernelGGL((attention_f32_kernel<E, 64>), grid, block, 0, ctx->stream, p);
  else if (p.dh <= 96) hipLaunchKernelGGL((attention_f32_kernel<E, 96>), grid, block, 0, ctx->stream, p);
  else hipLaunchKernelGGL((attention_f32_kernel<E, 128>), grid, block, 0, ctx->stream, p);
}

}  // namespace strp

using namespace strp;

extern "C" strp_status strp_attention(strp_ctx* ctx, const strp_attention_in* in) {
  if (!ctx) return STRP_EINVAL;
  if (!in || !in->Q || !in->K || !in->V || !in->C) return fail(ctx, STRP_EINVAL, "attention: null Q, K, V or C");
  if (!known_dtype(in->dtype)) return fail(ctx, STRP_EINVAL, "attention: unknown dtype");
  if (in->heads <= 0 || in->kv_heads <= 0 || in->d_head <= 0 || in->T <= 0) return fail(ctx, STRP_EINVAL, "attention: heads, kv_heads, d_head and T must be positive");
  if (in->d_head > 128) return fail(ctx, STRP_EINVAL, "attention: d_head above 128");
  if (in->heads > 65535) return fail(ctx, STRP_EINVAL, "attention: more than 65535 heads");
  if (!in->kv_of_head && in->heads % in->kv_heads) return fail(ctx, STRP_EINVAL, "attention: kv_heads does not divide heads and kv_of_head is null");
  if (in->n_seq < 0 || (in->seq_start ? in->n_seq < 1 : in->n_seq != 0)) return fail(ctx, STRP_EINVAL, "attention: seq_start needs n_seq > 0, no seq_start n_seq = 0");
  if (!(in->scale > 0.0f) || std::isinf(in->scale)) return fail(ctx, STRP_EINVAL, "attention: scale must be positive and finite");
  if (!token_ld(in->ldq, in->T) || !token_ld(in->ldk, in->T) || !token_ld(in->ldv, in->T) || !token_ld(in->ldc, in->T))
    return fail(ctx, STRP_EINVAL, "attention: leading dimensions must be multiples of 8 and not below T");
  if (!ptr16(in->Q) || !ptr16(in->K) || !ptr16(in->V) || !ptr16(in->C)) return fail(ctx, STRP_EINVAL, "attention: Q, K, V or C not 16-byte aligned");
  if (in->T > 0x7fffff00LL) return fail(ctx, STRP_EINVAL, "attention: T does not fit 31 bits");
  OnDevice on(ctx);
  if (!on.ok()) return fail(ctx, STRP_EHIP, "attention: device %d cannot be made current", ctx->device);
  AttnP p{in->Q, in->K, in->V, in->C, in->seq_start, in->kv_of_head, in->heads, in->kv_heads, in->heads / in->kv_heads, in->d_head, in->n_seq,
          (int)((in->T + 127) / 128), in->T, in->ldq, in->ldk, in->ldv, in->ldc, in->scale * 1.44269504088896341f};
  if (p.group == 0) p.group = 1;
  // the lengths are on the device: the operations of one sequence of all tokens
  const double T = (double)in->T;
  ProfScope ps(ctx, "attention", 2.0 * in->heads * in->d_head * T * (T + 1.0), bytes_of(in->dtype) * T * in->d_head * 2.0 * (in->heads + in->kv_heads));
  if (in->dtype == STRP_BF16) launch_attention_f32<__bf16>(ctx, p);
  else launch_attention_f32<float>(ctx, p);
  STRP_HIP(ctx, hipGetLastError());
  return STRP_OK;
}
