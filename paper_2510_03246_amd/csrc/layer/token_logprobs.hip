// Log probabilities of given tokens, entropy and best alternatives from logits [V x T], tokens contiguous.
//
// With m the maximum of a token's logits, e_v = (x_v - m) log2(e), s = sum 2^e_v and u = sum 2^e_v e_v:
//   log p_y = x_y - m - ln s,   entropy = ln s - ln2 u / s.
// (m, s, u) of a part of the vocabulary and of another merge into those of both, so one pass over the logits is enough.
//
// The vocabulary is cut into streams of L consecutive entries, a thread each (16 bytes of tokens wide).  The k best entries of a token
// lie in the k streams with the best maxima (an entry outside them has k streams with something better before it), equal ones in the
// order of the streams; so the pass over the logits keeps the maximum of every stream only, and the second kernel
// looks for the alternatives among k L entries.  50000 entries of 2048 tokens in bf16: 87 us, the first kernel about 50 of them at 4 TB/s, which memory bounds; one token 20 us, latencies.
#include "layer_ops.h"

#include <cmath>
#include <type_traits>

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
  floatx4* part;     // [tp][slices] m, s, u
  float* tops;       // [tp][lanes] maxima of the streams, null: not wanted
  int lanes;         // streams rounded up to whole slices
};

template <typename E>
__global__ __launch_bounds__(256) void logit_streams_kernel(const LogitP p) {
  constexpr int VEC = 16 / sizeof(E), UN = 8;
  __shared__ Soft sh[256][VEC];
  __shared__ float turned[64 * 33];        // ct VEC tokens x (rl + 1)
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
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) sh[threadIdx.x][e] = a[e];
  if (p.tops) {
    // a token's maxima lie side by side, as the kernel that reads them wants them; strides of powers of two between them would all meet in one channel of memory
#pragma unroll
    for (int e = 0; e < VEC; ++e) turned[(c * VEC + e) * (rl + 1) + r] = a[e].m;
    __syncthreads();
    const long long first = (long long)blockIdx.x * p.ct * VEC;
    const int bits = 31 - __clz(rl);
    for (int i = threadIdx.x; i < p.ct * VEC * rl; i += 256) {
      const int tok = i >> bits, st = i & (rl - 1);
      if (first + tok < p.T) p.tops[(first + tok) * p.lanes + (int)blockIdx.y * rl + st] = turned[tok * (rl + 1) + st];
    }
  }
  for (int o = rl >> 1; o > 0; o >>= 1) {
    __syncthreads();
    if (r < o)
#pragma unroll
      for (int e = 0; e < VEC; ++e) sh[threadIdx.x][e] = merge(sh[threadIdx.x][e], sh[threadIdx.x + o * p.ct][e]);
  }
  if (r == 0)
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (t0 + e < p.T) p.part[(t0 + e) * p.slices + blockIdx.y] = floatx4{sh[c][e].m, sh[c][e].s, sh[c][e].u, 0.0f};
}

// Maximum over the wavefront, in every lane.
__device__ __forceinline__ float wave_max(float v) {
  const auto step = [&](auto ctl) {
    const int o = __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, -INFINITY), __builtin_bit_cast(int, v), decltype(ctl)::value, 0xf, 0xf, false);
    v = fmaxf(v, __builtin_bit_cast(float, o));
  };
  step(std::integral_constant<int, 0x111>());      // row_shr 1, 2, 4, 8: the last lane of a row of 16 has its maximum
  step(std::integral_constant<int, 0x112>());
  step(std::integral_constant<int, 0x114>());
  step(std::integral_constant<int, 0x118>());
  step(std::integral_constant<int, 0x142>());      // row_bcast 15, 31: and lane 63 that of all
  step(std::integral_constant<int, 0x143>());
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// Candidates 0 .. limit - 1 with values f, none of them NaN; lane j < count holds the start of a block of B of them (a power of two), ascending.  Afterwards it
// holds the j-th of the k best candidates: ascending, or by rank where `by_rank` (equal ones: the lower first), its value in v.  A round cuts the blocks
// into 64 runs, one a lane, and keeps the k runs with the best maxima: no other run has a candidate that k others are not ahead of.  Runs of up to 8 stay in
// registers and give their candidates at once.
struct Best {
  int at;
  float v;
  int count;
};
template <typename F>
__device__ __forceinline__ void narrow(Best& b, int B, int limit, int k, bool by_rank, F f) {
  constexpr int R = 8;
  const int lane = threadIdx.x & 63;
  while (true) {
    int blocks = 1;
    while (blocks < b.count) blocks <<= 1;
    const int r = B * blocks > 64 ? B * blocks >> 6 : 1, runs = B / r, j = lane / runs, at = __shfl(b.at, j & 63, 64) + (lane - j * runs) * r;
    const bool there = j < b.count && at < limit;
    const int n = there ? min(r, limit - at) : 0;       // candidates of this lane
    if (r > R) {
      float v = -INFINITY;
      for (int i = 0; i < r; i += 8) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = f(there ? at + min(i + e, n - 1) : 0);
#pragma unroll
        for (int e = 0; e < 8; ++e) v = fmaxf(v, x[e]);
      }
      bool alive = there;
      int c = 0;
#pragma unroll 1
      for (; c < k; ++c) {
        const float m = wave_max(alive ? v : -INFINITY);
        const unsigned long long who = __ballot(alive && v == m);
        if (!who) break;
        if (lane == __ffsll((long long)who) - 1) alive = false;
      }
      const unsigned long long mask = __ballot(there && !alive);
      const int place = there && !alive ? __popcll(mask & ((1ull << lane) - 1)) : 63;      // k is below 63: that lane's is not used
      b.at = __builtin_amdgcn_ds_permute(4 * place, at);
      b.count = c;
      B = r;
      continue;
    }
    // what is taken, or is no candidate, is NaN: no maximum, and equal to none
    float x[R];
#pragma unroll
    for (int e = 0; e < R; ++e) {
      const float v = f(n ? at + min(e, n - 1) : 0);
      x[e] = e < n ? v : NAN;
    }
    int c = 0, my_at = 0;
    float my_v = 0.0f;
#pragma unroll 1
    for (; c < k; ++c) {
      float v = x[0];
#pragma unroll
      for (int e = 1; e < R; ++e) v = fmaxf(v, x[e]);
      const float m = wave_max(v);
      const unsigned long long who = __ballot(v == m);
      if (!who) break;
      const int from = __ffsll((long long)who) - 1;
      int best = 0;
#pragma unroll
      for (int e = R - 1; e >= 0; --e) best = x[e] == m ? e : best;
      const int at_best = __builtin_amdgcn_readlane(at + best, from);
      if (lane == c) {
        my_at = at_best;
        my_v = m;
      }
      best = lane == from ? best : R;
#pragma unroll
      for (int e = 0; e < R; ++e) x[e] = e == best ? NAN : x[e];
    }
    if (!by_rank) {                                     // ascending
      int place = 0;
      for (int e = 0; e < c; ++e) place += __builtin_amdgcn_readlane(my_at, e) < my_at;
      my_at = __builtin_amdgcn_ds_permute(4 * (lane < c ? place : 63), my_at);
    }
    b.at = my_at;
    b.v = my_v;
    b.count = c;
    return;
  }
}

struct TokenP {
  const void* logits;
  int V;
  long long T, ldl;
  int L, streams, slices;
  const floatx4* part;
  const float* tops;
  int lanes;
  const int32_t* target;
  float* logp;
  float* entropy;
  int k;
  int32_t* top_id;
  float* top_logp;
  long long ldt;
};

// Sixteen wavefronts have 16 / WPT neighbouring tokens (which share the lines of memory that they read), WPT wavefronts a token: all of them look
// for the best of the streams' maxima, the first for the alternatives in the streams.  What bounds it is the latency of the reads that follow each other.
template <typename E, int WPT>
__global__ __launch_bounds__(1024) void token_finish_kernel(const TokenP p) {
  constexpr int TOK = 16 / WPT;
  __shared__ Soft softs[16];
  __shared__ float runs[16 * 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = wave % WPT, token = wave / WPT;
  const long long t0 = (long long)blockIdx.x * TOK + token, t = t0 < p.T ? t0 : p.T - 1;
  const E* x = (const E*)p.logits + t;
  const float* tops = p.tops + t * p.lanes;
  const int y = p.logp ? p.target[t] : -1;
  const float xy = y >= 0 && y < p.V ? (float)x[(long long)y * p.ldl] : 0.0f;
  // a lane has B streams
  int B = 1;
  while (B * 64 * WPT < p.streams) B <<= 1;
  float run = -INFINITY;
  if (p.k) {
    const int s0 = (part * 64 + lane) * B;
    for (int i = 0; i < B; i += 8) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = tops[min(s0 + min(i + e, B - 1), p.streams - 1)];
#pragma unroll
      for (int e = 0; e < 8; ++e) run = fmaxf(run, v[e]);
    }
    if (WPT > 1) runs[(token * WPT + part) * 64 + lane] = run;
  }
  Soft a{-INFINITY, 0.0f, 0.0f};
  for (int s = part * 64 + lane; s < p.slices; s += 64 * WPT) {
    const floatx4 q = p.part[t * p.slices + s];
    a = merge(a, Soft{q[0], q[1], q[2]});
  }
#pragma unroll 1
  for (int o = 1; o < 64; o <<= 1) a = merge(a, Soft{__shfl_xor(a.m, o, 64), __shfl_xor(a.s, o, 64), __shfl_xor(a.u, o, 64)});
  if (WPT > 1) {
    if (lane == 0) softs[wave] = a;
    __syncthreads();
    if (part != 0) return;
    for (int w = 1; w < WPT; ++w) a = merge(a, softs[token * WPT + w]);
  }
  if (t0 >= p.T) return;
  const float log_s = logf(a.s);
  if (lane == 0) {
    if (p.logp) p.logp[t] = y >= 0 && y < p.V ? (xy - a.m) - log_s : 0.0f;
    if (p.entropy) p.entropy[t] = log_s - LN2 * a.u / a.s;
  }
  if (p.k == 0) return;
  if (!(a.m == a.m)) {
    if (lane < p.k) {
      p.top_id[(long long)lane * p.ldt + t] = -1;
      p.top_logp[(long long)lane * p.ldt + t] = NAN;
    }
    return;
  }
  // the best runs of streams, of those the best streams, of those the best entries
  Best b{0, 0.0f, 1};
  const int n_runs = (p.streams + B - 1) / B;
  narrow(b, 64 * WPT, n_runs, p.k, false, [&](int i) { return WPT > 1 ? runs[token * WPT * 64 + i] : __shfl(run, i, 64); });
  b.at *= B;
  narrow(b, B, p.streams, p.k, false, [&](int i) { return tops[i]; });
  b.at *= p.L;
  narrow(b, p.L, p.V, p.k, true, [&](int i) { return (float)x[(long long)i * p.ldl]; });
  if (lane < p.k) {
    p.top_id[(long long)lane * p.ldt + t] = b.at;
    p.top_logp[(long long)lane * p.ldt + t] = (b.v - a.m) - log_s;
  }
}

template <typename E>
static void launch_logprobs(strp_ctx* ctx, const LogitP& a, const TokenP& b) {
  const long long cols = a.ct * (16 / (long long)sizeof(E));
  hipLaunchKernelGGL((logit_streams_kernel<E>), dim3((unsigned)((a.T + cols - 1) / cols), a.slices), dim3(256), 0, ctx->stream, a);
  // Eight wavefronts for a token, one where the tokens alone are wavefronts enough.  Both kernels, us, 50000 entries of bf16, one against eight: one token 57, 24; 512 86, 41; 2048 89, 85;
  // 4096 150, 162; 8192 287, 310.  (Four: 2048 86.5; sixteen: one token 23, 512 51.)  Measured at these sizes alone: 130000 entries over 2048 tokens in eight 175, over 2100 in one 219.
  const auto go = [&](auto kernel, int tokens) { hipLaunchKernelGGL(kernel, dim3((unsigned)((b.T + tokens - 1) / tokens)), dim3(1024), 0, ctx->stream, b); };
  if (b.T <= 2048) go(token_finish_kernel<E, 8>, 2);
  else go(token_finish_kernel<E, 1>, 16);
}

// How a vocabulary is cut.
struct LogitPlan {
  int ct, L, streams, slices, lanes;
  size_t part_bytes, tops_bytes;
};
static LogitPlan plan_logits(int V, long long T, int dtype) {
  LogitPlan q;
  const long long vec = 16 / (long long)bytes_of(dtype), chunks = (T + vec - 1) / vec;
  q.ct = 1;
  while (q.ct < 8 && q.ct < chunks) q.ct *= 2;
  // streams of 8, 16 or 32 entries (a power of two): long where the tokens alone fill the chip, since every stream leaves a maximum behind
  const long long want = 262144 / chunks > 0 ? 262144 / chunks : 1;
  int L = 8;
  while (L < 32 && 2 * L * want <= V) L *= 2;
  const int rl = 256 / q.ct;
  // at most 65535 slices
  while (((V + L - 1) / L + rl - 1) / rl > 65535) L *= 2;
  q.L = L;
  q.streams = (int)((V + L - 1) / L);
  q.slices = (q.streams + rl - 1) / rl;
  q.lanes = q.slices * rl;
  q.part_bytes = (size_t)T * q.slices * 16;
  q.tops_bytes = (size_t)T * q.lanes * 4;
  return q;
}
static size_t up256(size_t b) { return (b + 255) & ~size_t(255); }

}  // namespace strp

using namespace strp;

extern "C" {

size_t strp_token_logprobs_workspace_bytes(int32_t V, int64_t T, int32_t n_top) {
  if (V <= 0 || V > (1 << 30) || T <= 0 || T > (1LL << 25) || n_top < 0) return 0;
  size_t most = 0;
  for (int dt : {STRP_BF16, STRP_F32}) {
    const LogitPlan q = plan_logits(V, T, dt);
    const size_t b = up256(q.part_bytes) + (n_top ? up256(q.tops_bytes) : 0) + 256;
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
  if (T > (1LL << 25) || V > (1 << 30)) return fail(ctx, STRP_EINVAL, "token_logprobs: more than 2^25 tokens or 2^30 entries");
  if (!ctx->ws) return fail(ctx, STRP_ENOMEM, "token_logprobs: no workspace set");
  const LogitPlan q = plan_logits(V, T, dtype);
  Arena arena(ctx);
  STRP_TAKE(ctx, arena, part, floatx4, q.part_bytes / 16);
  float* tops = nullptr;
  if (n_top) {
    STRP_TAKE(ctx, arena, maxima, float, q.tops_bytes / 4);
    tops = maxima;
  }
  OnDevice on(ctx);
  if (!on.ok()) return fail(ctx, STRP_EHIP, "token_logprobs: device %d cannot be made current", ctx->device);
  ProfScope ps(ctx, "token_logprobs", 6.0 * V * (double)T, bytes_of(dtype) * (double)V * (double)T);
  const LogitP a{logits, V, T, ldl, q.ct, q.L, q.streams, q.slices, part, tops, q.lanes};
  const TokenP b{logits, V, T, ldl, q.L, q.streams, q.slices, part, tops, q.lanes, target, logp, entropy, n_top, top_id, top_logp, ldt};
  if (dtype == STRP_BF16) launch_logprobs<__bf16>(ctx, a, b);
  else launch_logprobs<float>(ctx, a, b);
  STRP_HIP(ctx, hipGetLastError());
  return STRP_OK;
}

}  // extern "C"
