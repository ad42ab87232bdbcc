// Log probabilities of given tokens, entropy and best alternatives from logits [V x T], tokens contiguous.
//
// With m the maximum of a token's logits, e_v = (x_v - m) log2(e), s = sum 2^e_v and u = sum 2^e_v e_v:
//   log p_y = x_y - m - ln s,   entropy = ln s - ln2 u / s.
// (m, s, u) of a part of the vocabulary and of another merge into those of both, so one pass over the logits is enough.
//
// The vocabulary is cut into streams of L consecutive entries, a thread each (16 bytes of tokens wide).  The k best entries of a token
// lie in the k streams with the best maxima (an entry outside them has k streams with something better before it), equal ones in the
// order of the streams; so the pass over the logits keeps the maximum of every stream only, and the second kernel
// looks for the alternatives among k L entries.
#include "layer_ops.h"

#include <cmath>

namespace strp {

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.69314718055994531f;
constexpr float FAR_BELOW = -16384.0f;       // a power of two that is zero; the logarithm of zero is held to it, so that 0 x -inf does not arise

struct Soft { float m, s, u; };

__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.0f : m; }
__device__ __forceinline__ float held(float e) { return __builtin_elementwise_maximum(e, FAR_BELOW); }      // NaN stays NaN
__device__ __forceinline__ void rescale(Soft& a, float ref) {
  const float d = held((a.m - ref) * LOG2E), f = __builtin_amdgcn_exp2f(d);
  a.u = (a.u + a.s * d) * f;
  a.s *= f;
}
__device__ __forceinline__ Soft merge(Soft a, Soft b) {
  const float m = __builtin_elementwise_maximum(a.m, b.m), ref = reference(m);
  rescale(a, ref);
  rescale(b, ref);
  return Soft{m, a.s + b.s, a.u + b.u};
}

struct LogitP {
  const void* logits;
  int V;
  long long T, ldl;
  int ct;            // 16-byte columns of a workgroup, a power of two
  int L, streams, slices;
  float* part;       // [slices][3][tp]
  float* tops;       // [streams][tp] maxima, null: not wanted
  long long tp;
};

template <typename E>
__global__ __launch_bounds__(256) void logit_streams_kernel(const LogitP p) {
  constexpr int VEC = 16 / sizeof(E), UN = 8;
  __shared__ Soft sh[256][VEC];
  const int c = threadIdx.x % p.ct, r = threadIdx.x / p.ct, rl = 256 / p.ct;
  const long long t0 = ((long long)blockIdx.x * p.ct + c) * VEC;
  const int stream = (int)blockIdx.y * rl + r;
  const bool in = t0 < p.T && stream < p.streams;
  Soft a[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) a[e] = Soft{-INFINITY, 0.0f, 0.0f};
  if (in) {
    const int v0 = stream * p.L, n = min(p.L, p.V - v0);
    const E* x = (const E*)p.logits + (long long)v0 * p.ldl + t0;
    auto take = [&](const float (&v)[VEC]) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float t = held((v[e] - reference(a[e].m)) * LOG2E), f = __builtin_amdgcn_exp2f(t);
        a[e].s += f;
        a[e].u += f * t;
      }
    };
    int i = 0;
    for (; i + UN <= n; i += UN) {
      float v[UN][VEC];
#pragma unroll
      for (int k = 0; k < UN; ++k) load_floats<VEC>(x + (long long)(i + k) * p.ldl, v[k]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        float m = a[e].m;
#pragma unroll
        for (int k = 0; k < UN; ++k) m = __builtin_elementwise_maximum(m, v[k][e]);
        rescale(a[e], reference(m));
        a[e].m = m;
      }
#pragma unroll
      for (int k = 0; k < UN; ++k) take(v[k]);
    }
    for (; i < n; ++i) {
      float v[VEC];
      load_floats<VEC>(x + (long long)i * p.ldl, v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float m = __builtin_elementwise_maximum(a[e].m, v[e]);
        rescale(a[e], reference(m));
        a[e].m = m;
      }
      take(v);
    }
    if (p.tops)
#pragma unroll
      for (int e = 0; e < VEC; ++e) p.tops[(long long)stream * p.tp + t0 + e] = a[e].m;
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) sh[threadIdx.x][e] = a[e];
  for (int o = rl >> 1; o > 0; o >>= 1) {
    __syncthreads();
    if (r < o)
#pragma unroll
      for (int e = 0; e < VEC; ++e) sh[threadIdx.x][e] = merge(sh[threadIdx.x][e], sh[threadIdx.x + o * p.ct][e]);
  }
  if (r == 0 && t0 < p.T)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      float* out = p.part + (long long)blockIdx.y * 3 * p.tp + t0 + e;
      out[0] = sh[c][e].m;
      out[p.tp] = sh[c][e].s;
      out[2 * p.tp] = sh[c][e].u;
    }
}

// The best k of what a wavefront has been shown: lane i < k holds the i-th, in descending order of the values and, among equal
// ones, ascending order of the indices.  NaN ranks nowhere.
struct TopList {
  float v;
  int at;
  __device__ TopList() : v(-INFINITY), at(0x7fffffff) {}
  __device__ __forceinline__ void show(float x, int i, bool valid, int k) {
    const int lane = threadIdx.x & 63;
    bool waits = valid;
    while (true) {
      const float lv = __shfl(v, k - 1, 64);
      const int li = __shfl(at, k - 1, 64);
      waits = waits && (x > lv || (x == lv && i < li));
      const unsigned long long who = __ballot(waits);
      if (!who) return;
      const int from = __ffsll((long long)who) - 1;
      const float nv = __shfl(x, from, 64);
      const int ni = __shfl(i, from, 64);
      const int place = __popcll(__ballot(lane < k && (v > nv || (v == nv && at < ni))));
      const float uv = __shfl_up(v, 1, 64);
      const int ui = __shfl_up(at, 1, 64);
      if (lane == place) { v = nv; at = ni; }
      else if (lane > place) { v = uv; at = ui; }
      if (lane == from) waits = false;
    }
  }
};

struct TokenP {
  const void* logits;
  int V;
  long long T, ldl;
  int L, streams, slices;
  const float* part;
  const float* tops;
  long long tp;
  const int32_t* target;
  float* logp;
  float* entropy;
  int k;
  int32_t* top_id;
  float* top_logp;
  long long ldt;
};

// A token has a wavefront.
template <typename E>
__global__ __launch_bounds__(256) void token_finish_kernel(const TokenP p) {
  const int lane = threadIdx.x & 63;
  const long long t = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= p.T) return;
  Soft a{-INFINITY, 0.0f, 0.0f};
  for (int s = lane; s < p.slices; s += 64) {
    const float* q = p.part + (long long)s * 3 * p.tp + t;
    a = merge(a, Soft{q[0], q[p.tp], q[2 * p.tp]});
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) a = merge(a, Soft{__shfl_xor(a.m, o, 64), __shfl_xor(a.s, o, 64), __shfl_xor(a.u, o, 64)});
  const float log_s = logf(a.s);
  const E* x = (const E*)p.logits + t;
  if (lane == 0) {
    if (p.logp) {
      const int y = p.target[t];
      p.logp[t] = y >= 0 && y < p.V ? ((float)x[(long long)y * p.ldl] - a.m) - log_s : 0.0f;
    }
    if (p.entropy) p.entropy[t] = log_s - LN2 * a.u / a.s;
  }
  if (p.k == 0) return;
  TopList where, best;
  for (int s = 0; s < p.streams; s += 64) {
    const int i = s + lane;
    where.show(i < p.streams ? p.tops[(long long)i * p.tp + t] : 0.0f, i, i < p.streams, p.k);
  }
  for (int e = 0; e < p.k * p.L; e += 64) {
    const int i = e + lane, st = i / p.L < p.k ? __shfl(where.at, i / p.L < p.k ? i / p.L : 0, 64) : __shfl(where.at, 0, 64);
    const long long v = (long long)st * p.L + i % p.L;
    const bool ok = i < p.k * p.L && st != 0x7fffffff && v < p.V;
    best.show(ok ? (float)x[v * p.ldl] : 0.0f, (int)v, ok, p.k);
  }
  if (lane < p.k) {
    const bool nan = !(a.m == a.m) || best.at == 0x7fffffff;
    p.top_id[(long long)lane * p.ldt + t] = nan ? -1 : best.at;
    p.top_logp[(long long)lane * p.ldt + t] = nan ? NAN : (best.v - a.m) - log_s;
  }
}

// How a vocabulary is cut.
struct LogitPlan {
  int ct, L, streams, slices;
  long long tp;
};
static LogitPlan plan_logits(int V, long long T, int dtype) {
  LogitPlan q;
  const long long vec = 16 / (long long)bytes_of(dtype), chunks = (T + vec - 1) / vec;
  q.tp = chunks * vec;
  q.ct = 1;
  while (q.ct < 8 && q.ct < chunks) q.ct *= 2;
  // streams of 8 to 32 entries: long where the tokens alone fill the chip, since every stream leaves a maximum behind
  const long long want = 262144 / chunks > 0 ? 262144 / chunks : 1;
  long long L = V / want / 8 * 8;
  L = L < 8 ? 8 : (L > 32 ? 32 : L);
  const int rl = 256 / q.ct;
  // at most 65535 slices
  while (((V + L - 1) / L + rl - 1) / rl > 65535) L *= 2;
  q.L = (int)L;
  q.streams = (int)((V + L - 1) / L);
  q.slices = (q.streams + rl - 1) / rl;
  return q;
}
static size_t up256(size_t b) { return (b + 255) & ~size_t(255); }

}  // namespace strp

using namespace strp;

extern "C" {

size_t strp_token_logprobs_workspace_bytes(int32_t V, int64_t T, int32_t n_top) {
  if (V <= 0 || T <= 0 || n_top < 0) return 0;
  size_t most = 0;
  for (int dt : {STRP_BF16, STRP_F32}) {
    const LogitPlan q = plan_logits(V, T, dt);
    const size_t b = up256((size_t)q.slices * 3 * q.tp * 4) + (n_top ? up256((size_t)q.streams * q.tp * 4) : 0) + 256;
    most = b > most ? b : most;
  }
  return most < 4096 ? 4096 : most;
}

strp_status strp_token_logprobs(strp_ctx* ctx, const void* logits, strp_dtype dtype, int32_t V, int64_t T, int64_t ldl, const int32_t* target,
                                float* logp, float* entropy, int32_t n_top, int32_t* top_id, float* top_logp, int64_t ldt) {
  if (!ctx) return STRP_EINVAL;
  if (!logits) return fail(ctx, STRP_EINVAL, "token_logprobs: null logits");
  if (!known_dtype(dtype)) return fail(ctx, STRP_EINVAL, "token_logprobs: unknown dtype");
  if (V <= 0 || T <= 0) return fail(ctx, STRP_EINVAL, "token_logprobs: V and T must be positive");
  if (n_top < 0 || n_top > STRP_TOP_MAX || n_top > V) return fail(ctx, STRP_EINVAL, "token_logprobs: n_top outside [0, min(V, %d)]", STRP_TOP_MAX);
  if ((target == nullptr) != (logp == nullptr)) return fail(ctx, STRP_EINVAL, "token_logprobs: target and logp belong together");
  if (n_top > 0 && (!top_id || !top_logp || ldt < T)) return fail(ctx, STRP_EINVAL, "token_logprobs: n_top > 0 needs top_id and top_logp with ldt >= T");
  if (!logp && !entropy && n_top == 0) return fail(ctx, STRP_EINVAL, "token_logprobs: nothing asked for");
  if (!token_ld(ldl, T)) return fail(ctx, STRP_EINVAL, "token_logprobs: ldl must be a multiple of 8 and not below T");
  if (!ptr16(logits)) return fail(ctx, STRP_EINVAL, "token_logprobs: logits not 16-byte aligned");
  if (T > (1LL << 31)) return fail(ctx, STRP_EINVAL, "token_logprobs: more than 2^31 tokens");
  if (!ctx->ws) return fail(ctx, STRP_ENOMEM, "token_logprobs: no workspace set");
  const LogitPlan q = plan_logits(V, T, dtype);
  Arena arena(ctx);
  STRP_TAKE(ctx, arena, part, float, (size_t)q.slices * 3 * q.tp);
  float* tops = nullptr;
  if (n_top) {
    STRP_TAKE(ctx, arena, maxima, float, (size_t)q.streams * q.tp);
    tops = maxima;
  }
  OnDevice on(ctx);
  if (!on.ok()) return fail(ctx, STRP_EHIP, "token_logprobs: device %d cannot be made current", ctx->device);
  ProfScope ps(ctx, "token_logprobs", 6.0 * V * (double)T, bytes_of(dtype) * (double)V * (double)T);
  const LogitP a{logits, V, T, ldl, q.ct, q.L, q.streams, q.slices, part, tops, q.tp};
  const TokenP b{logits, V, T, ldl, q.L, q.streams, q.slices, part, tops, q.tp, target, logp, entropy, n_top, top_id, top_logp, ldt};
  const long long cols = q.ct * (16 / (long long)bytes_of(dtype));
  const dim3 grid((unsigned)((T + cols - 1) / cols), q.slices), finish((unsigned)((T + 3) / 4)), block(256);
  if (dtype == STRP_BF16) {
    hipLaunchKernelGGL((logit_streams_kernel<__bf16>), grid, block, 0, ctx->stream, a);
    hipLaunchKernelGGL((token_finish_kernel<__bf16>), finish, block, 0, ctx->stream, b);
  } else {
    hipLaunchKernelGGL((logit_streams_kernel<float>), grid, block, 0, ctx->stream, a);
    hipLaunchKernelGGL((token_finish_kernel<float>), finish, block, 0, ctx->stream, b);
  }
  STRP_HIP(ctx, hipGetLastError());
  return STRP_OK;
}

}  // extern "C"
