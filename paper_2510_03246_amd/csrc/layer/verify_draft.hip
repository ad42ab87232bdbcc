// Drafted tokens against the target's probabilities, and the token that follows them.
//
//   keep x where u q(x) < p(x);  then the lowest v with sum_{w <= v} r(w) > u' sum r,  r = max(p - q, 0) or p,
// with p and q the softmax of two columns of logits [V x tokens].  What is asked is an index into 10^5 sums, of which some lie within 10^-7 of each other:
// 32 bits would answer beside it once in a few hundred times, so exponentials and sums are of 64.
//
// Three kernels: sums of exponentials of slices of every column; the sequences' first token that is not kept and the sums of r over
// parts of the vocabulary; the part that holds the answer, entry by entry.
#include "layer_ops.h"

namespace strp {

constexpr int SLICES = 64, PARTS = 64;     // at most: a wavefront has one of each a lane

// e^y in 64 bits for y <= 600, 0 where y is below -745 (NaN: 0 too): 2^k e^r with |r| <= ln 2 / 2, the series to r^12 (the next term is below 2e-16)
__device__ __forceinline__ double exp64(double y) {
  y = fmax(y, -800.0);
  const double k = __builtin_rint(y * 1.4426950408889634074);
  double r = __builtin_fma(-k, 6.93147180369123816490e-01, y);      // ln 2 in two parts, the first of 32 bits: its product with k is exact
  r = __builtin_fma(-k, 1.90821492927058770002e-10, r);
  double p = 1.0 / 479001600.0;
  p = __builtin_fma(p, r, 1.0 / 39916800.0);
  p = __builtin_fma(p, r, 1.0 / 3628800.0);
  p = __builtin_fma(p, r, 1.0 / 362880.0);
  p = __builtin_fma(p, r, 1.0 / 40320.0);
  p = __builtin_fma(p, r, 1.0 / 5040.0);
  p = __builtin_fma(p, r, 1.0 / 720.0);
  p = __builtin_fma(p, r, 1.0 / 120.0);
  p = __builtin_fma(p, r, 1.0 / 24.0);
  p = __builtin_fma(p, r, 1.0 / 6.0);
  p = __builtin_fma(p, r, 0.5);
  p = __builtin_fma(p, r, 1.0);
  p = __builtin_fma(p, r, 1.0);
  return __builtin_ldexp(p, (int)k);
}

// Sum of e^((x - ref) / temperature) over some entries.  ref is one of them and no more than 500 temperatures below any: with 64 bits it need not be the largest.
// most: the largest, NaN where there is one.
struct __attribute__((aligned(16))) Mass {
  double sum;
  float ref, most;
};

struct VerifyP {
  const void* target;
  const void* draft;
  const int32_t* draft_id;
  const float* u;
  const float* u_next;
  const int32_t* draft_start;
  int32_t* accepted;
  int32_t* next_id;
  int V, n_seq, T, columns;                // columns of the target: T + n_seq
  long long ldt, ldd;
  double inv;                              // 1 / temperature
  int ct, groups_t, slices, rows;          // first kernel: 16-byte columns a workgroup, workgroups across the target, slices of `rows` entries
  Mass* mass;                              // [columns + T][slices]
  int parts, part_rows;
  struct Chosen* chosen;                   // [n_seq]
  double* sums;                            // [n_seq][parts][2] of r and of p
};

// the column of p, that of q (-1: none), and what makes probabilities of exponentials; bad: no answer
struct Chosen { int col_t, col_d, bad, pad; double ref_t, inv_t, ref_d, inv_d; };

__device__ __forceinline__ Mass joined(Mass a, Mass b, double inv) {
  Mass r;
  r.ref = fmaxf(a.ref, b.ref);             // -inf where neither has an entry, and then both sums are zero
  r.most = __builtin_elementwise_maximum(a.most, b.most);
  r.sum = a.sum * (a.ref == r.ref ? 1.0 : exp64(((double)a.ref - (double)r.ref) * inv)) + b.sum * (b.ref == r.ref ? 1.0 : exp64(((double)b.ref - (double)r.ref) * inv));
  return r;
}

template <typename E>
__global__ __launch_bounds__(256) void verify_sums_kernel(const VerifyP p) {
  constexpr int VEC = 16 / sizeof(E);
  __shared__ Mass sh[256];
  const bool of_draft = (int)blockIdx.x >= p.groups_t;
  const int c = threadIdx.x % p.ct, r = threadIdx.x / p.ct, rl = 256 / p.ct;
  const long long t0 = ((long long)((int)blockIdx.x - (of_draft ? p.groups_t : 0)) * p.ct + c) * VEC, ld = of_draft ? p.ldd : p.ldt;
  const int n = of_draft ? p.T : p.columns, v0 = (int)blockIdx.y * p.rows, v1 = min(v0 + p.rows, p.V);
  Mass a[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) a[e] = Mass{0.0, -INFINITY, -INFINITY};
  if (t0 < n) {
    const E* x = (const E*)(of_draft ? p.draft : p.target) + t0;
    for (int v = v0 + r; v < v1; v += rl) {
      float f[VEC];
      load_floats<VEC>(x + (long long)v * ld, f);
      bool far = false;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        a[e].most = __builtin_elementwise_maximum(a[e].most, f[e]);
        far = far || (f[e] > a[e].ref && ((double)f[e] - (double)a[e].ref) * p.inv > 500.0);
      }
      if (far)
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (f[e] > a[e].ref && ((double)f[e] - (double)a[e].ref) * p.inv > 500.0) {
            a[e].sum *= exp64(((double)a[e].ref - (double)f[e]) * p.inv);
            a[e].ref = f[e];
          }
#pragma unroll
      for (int e = 0; e < VEC; ++e) a[e].sum += exp64(((double)f[e] - (double)a[e].ref) * p.inv);
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    __syncthreads();
    sh[threadIdx.x] = a[e];
    for (int o = rl >> 1; o > 0; o >>= 1) {
      __syncthreads();
      if (r < o) sh[threadIdx.x] = joined(sh[threadIdx.x], sh[threadIdx.x + o * p.ct], p.inv);
    }
    if (r == 0 && t0 + e < n) p.mass[(t0 + e + (of_draft ? p.columns : 0)) * p.slices + blockIdx.y] = sh[c];
  }
}

// All slices of a column, in every lane of the wavefront.
__device__ __forceinline__ Mass whole_column(const VerifyP& p, long long column) {
  const int lane = threadIdx.x & 63;
  Mass a = Mass{0.0, -INFINITY, -INFINITY};
  if (lane < p.slices) a = p.mass[column * p.slices + lane];
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    Mass b;
    b.sum = __shfl_xor(a.sum, o, 64);
    b.ref = __shfl_xor(a.ref, o, 64);
    b.most = __shfl_xor(a.most, o, 64);
    a = lane & o ? joined(b, a, p.inv) : joined(a, b, p.inv);      // the same in both lanes, to the bit
  }
  return a;
}

__device__ __forceinline__ double weight(const Chosen& c, float xt, float xd, bool rest, double inv) {
  const double pt = exp64(((double)xt - c.ref_t) * inv) * c.inv_t;
  if (!rest) return pt;
  return fmax(pt - exp64(((double)xd - c.ref_d) * inv) * c.inv_d, 0.0);
}

template <typename E>
__global__ __launch_bounds__(256) void verify_weigh_kernel(const VerifyP p) {
  __shared__ Chosen sc;
  __shared__ int stop[4];
  __shared__ Chosen found[4];
  __shared__ double sr[4], sp[4];
  const int seq = (int)blockIdx.x, part = (int)blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const auto begin = [&](int s) { return p.draft_start ? min(max(p.draft_start[s], 0), p.T) : (s ? p.T : 0); };
  const int a = begin(seq), n = max(begin(seq + 1) - a, 0);
  const E* target = (const E*)p.target;
  const E* draft = (const E*)p.draft;
  // the positions four at a time, a wavefront each: every part does so again, which costs less than a kernel of its own
  int accepted = n;
  for (int i0 = 0; i0 <= n; i0 += 4) {
    const int i = i0 + wave;
    if (i <= n) {
      const int ct = min(a + seq + i, p.columns - 1);
      const Mass mt = whole_column(p, ct);
      Chosen c = Chosen{ct, -1, 0, 0, (double)mt.ref, 1.0 / mt.sum, 0.0, 0.0};
      c.bad = !(fabsf(mt.most) < INFINITY);
      bool keep = false;
      if (i < n) {
        const Mass md = whole_column(p, (long long)p.columns + a + i);
        c.col_d = a + i;
        c.ref_d = md.ref;
        c.inv_d = 1.0 / md.sum;
        c.bad = c.bad || !(fabsf(md.most) < INFINITY);
        const int x = p.draft_id[a + i];
        if (x >= 0 && x < p.V && !c.bad) {
          const double pt = exp64(((double)(float)target[(long long)x * p.ldt + ct] - c.ref_t) * p.inv) * c.inv_t;
          const double qd = exp64(((double)(float)draft[(long long)x * p.ldd + a + i] - c.ref_d) * p.inv) * c.inv_d;
          keep = (double)p.u[a + i] * qd < pt;
        }
      }
      if (lane == 0) {
        stop[wave] = !keep;
        found[wave] = c;
      }
    }
    __syncthreads();
    int at = -1;
    for (int w = 3; w >= 0; --w)
      if (i0 + w <= n && stop[w]) at = w;
    if (at >= 0) {
      accepted = i0 + at;
      if (threadIdx.x == 0) sc = found[at];
      __syncthreads();
      break;
    }
    __syncthreads();
  }
  const Chosen c = sc;
  if (part == 0 && threadIdx.x == 0) {
    p.accepted[seq] = accepted;
    p.chosen[seq] = c;
  }
  const int v0 = part * p.part_rows, v1 = min(v0 + p.part_rows, p.V);
  double r = 0.0, s = 0.0;
  if (!c.bad)
    for (int v = v0 + (int)threadIdx.x; v < v1; v += 256) {
      const float xt = (float)target[(long long)v * p.ldt + c.col_t];
      const double pt = exp64(((double)xt - c.ref_t) * p.inv) * c.inv_t;
      s += pt;
      if (c.col_d >= 0) r += fmax(pt - exp64(((double)(float)draft[(long long)v * p.ldd + c.col_d] - c.ref_d) * p.inv) * c.inv_d, 0.0);
    }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    r += __shfl_xor(r, o, 64);
    s += __shfl_xor(s, o, 64);
  }
  if (lane == 0) {
    sr[wave] = r;
    sp[wave] = s;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double* to = p.sums + ((long long)seq * p.parts + part) * 2;
    to[0] = ((sr[0] + sr[1]) + sr[2]) + sr[3];
    to[1] = ((sp[0] + sp[1]) + sp[2]) + sp[3];
  }
}

// sum over the lanes up to this one
__device__ __forceinline__ double upto(double x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double y = __shfl_up(x, o, 64);
    x = lane >= o ? y + x : x;
  }
  return x;
}

template <typename E>
__global__ __launch_bounds__(256) void verify_find_kernel(const VerifyP p) {
  __shared__ double totals[4];
  __shared__ int firsts[4], lasts[4];
  const int seq = (int)blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Chosen c = p.chosen[seq];
  if (c.bad) {
    if (threadIdx.x == 0) p.next_id[seq] = -1;
    return;
  }
  // every wavefront finds the part for itself
  const double* from = p.sums + (long long)seq * p.parts * 2;
  const double r = lane < p.parts && c.col_d >= 0 ? from[2 * lane] : 0.0, s = lane < p.parts ? from[2 * lane + 1] : 0.0;
  const bool rest = __builtin_amdgcn_ballot_w64(r > 0.0) != 0;
  const double mine = rest ? r : s, sum = upto(mine), total = __shfl(sum, 63, 64);
  const float u = p.u_next[seq];
  const double goal = u < 1.0f ? (double)u * total : (double)INFINITY;
  const unsigned long long over = __builtin_amdgcn_ballot_w64(sum > goal && mine > 0.0), some = __builtin_amdgcn_ballot_w64(mine > 0.0);
  const int part = over ? __builtin_ctzll(over) : some ? 63 - __builtin_clzll(some) : 0;
  double before = __shfl(sum, part > 0 ? part - 1 : 0, 64);
  if (part == 0) before = 0.0;
  // its entries, 256 at a time
  const int v0 = part * p.part_rows, v1 = min(v0 + p.part_rows, p.V);
  int last = -1;                           // the last entry with r > 0, should rounding leave the sums of the part below the goal
  for (int b = v0; b < v1; b += 256) {
    const int v = b + (int)threadIdx.x;
    double w = 0.0;
    if (v < v1) w = weight(c, (float)((const E*)p.target)[(long long)v * p.ldt + c.col_t], rest ? (float)((const E*)p.draft)[(long long)v * p.ldd + c.col_d] : 0.0f, rest, p.inv);
    double run = upto(w);
    if (lane == 63) totals[wave] = run;
    __syncthreads();
    double base = before;
    for (int i = 0; i < wave; ++i) base += totals[i];
    run += base;
    const unsigned long long yes = __builtin_amdgcn_ballot_w64(w > 0.0 && run > goal), any = __builtin_amdgcn_ballot_w64(w > 0.0);
    if (lane == 0) {
      firsts[wave] = yes ? __builtin_ctzll(yes) + 64 * wave : -1;
      lasts[wave] = any ? 63 - __builtin_clzll(any) + 64 * wave : -1;
    }
    __syncthreads();
    int first = -1;
    for (int i = 3; i >= 0; --i) first = firsts[i] >= 0 ? firsts[i] : first;
    for (int i = 0; i < 4; ++i) last = lasts[i] >= 0 ? b + lasts[i] : last;
    if (first >= 0) {
      last = b + first;
      break;
    }
    before = ((before + totals[0]) + totals[1]) + totals[2] + totals[3];
    __syncthreads();
  }
  if (threadIdx.x == 0) p.next_id[seq] = last;
}

struct VerifyPlan {
  int ct, groups_t, groups_d, slices, rows, parts, part_rows;
};
static VerifyPlan plan_verify(int V, long long T, int n_seq, int dtype) {
  VerifyPlan q;
  const long long vec = dtype == STRP_BF16 ? 8 : 4, chunks_t = (T + n_seq + vec - 1) / vec, chunks_d = (T + vec - 1) / vec;
  const int widest = 8;                    // a line of 128 bytes
  q.ct = 1;
  while (q.ct < widest && q.ct < chunks_t) q.ct *= 2;
  q.groups_t = (int)((chunks_t + q.ct - 1) / q.ct);
  q.groups_d = (int)((chunks_d + q.ct - 1) / q.ct);
  // as many slices as fill the chip twice over, none below one entry a thread
  long long slices = 2048 / (q.groups_t + q.groups_d) + 1;
  const long long most = (V + 256 / q.ct - 1) / (256 / q.ct);
  if (slices > most) slices = most;
  if (slices > SLICES) slices = SLICES;
  q.rows = (int)((V + slices - 1) / slices);
  q.slices = (V + q.rows - 1) / q.rows;
  long long parts = (V + 255) / 256;
  if (parts > PARTS) parts = PARTS;
  q.part_rows = (int)((V + parts - 1) / parts);
  q.parts = (V + q.part_rows - 1) / q.part_rows;
  return q;
}
static size_t up256(size_t b) { return (b + 255) & ~size_t(255); }

template <typename E>
static void launch_verify(strp_ctx* ctx, const VerifyP& p, const VerifyPlan& q) {
  hipLaunchKernelGGL((verify_sums_kernel<E>), dim3((unsigned)(q.groups_t + q.groups_d), (unsigned)q.slices), dim3(256), 0, ctx->stream, p);
  hipLaunchKernelGGL((verify_weigh_kernel<E>), dim3((unsigned)p.n_seq, (unsigned)q.parts), dim3(256), 0, ctx->stream, p);
  hipLaunchKernelGGL((verify_find_kernel<E>), dim3((unsigned)p.n_seq), dim3(256), 0, ctx->stream, p);
}

}  // namespace strp

using namespace strp;

extern "C" {

size_t strp_verify_draft_workspace_bytes(int32_t V, int64_t T, int32_t n_seq) {
  if (V <= 0 || V > (1 << 30) || T < 0 || T > (1 << 20) || n_seq <= 0 || n_seq > 65536) return 0;
  // (a workspace has 4 KB at least)
  return 4096 + up256((size_t)(2 * T + n_seq) * SLICES * sizeof(Mass)) + up256((size_t)n_seq * sizeof(Chosen)) + up256((size_t)n_seq * PARTS * 16);
}

strp_status strp_verify_draft(strp_ctx* ctx, const strp_verify_draft_in* in) {
  if (!ctx) return STRP_EINVAL;
  if (!in || !in->target || !in->u_next || !in->accepted || !in->next_id) return fail(ctx, STRP_EINVAL, "verify_draft: null target, u_next, accepted or next_id");
  if (!known_dtype(in->dtype)) return fail(ctx, STRP_EINVAL, "verify_draft: unknown dtype");
  if (in->V <= 0 || in->n_seq <= 0 || in->T < 0) return fail(ctx, STRP_EINVAL, "verify_draft: V and n_seq must be positive, T not negative");
  if (in->T > 0 && (!in->draft || !in->draft_id || !in->u)) return fail(ctx, STRP_EINVAL, "verify_draft: T > 0 needs draft, draft_id and u");
  if (in->V > (1 << 30) || in->T > (1 << 20) || in->n_seq > 65536)
    return fail(ctx, STRP_EINVAL, "verify_draft: V above 2^30, T above 2^20 or n_seq above 65536");
  if (!in->draft_start && in->n_seq != 1 && in->T > 0) return fail(ctx, STRP_EINVAL, "verify_draft: no draft_start needs n_seq = 1 or T = 0");
  if (!(in->temperature >= 1e-30) || !(in->temperature <= 1e30)) return fail(ctx, STRP_EINVAL, "verify_draft: temperature must be from 1e-30 to 1e30");
  if (!token_ld(in->ldt, in->T + in->n_seq) || (in->T > 0 && !token_ld(in->ldd, in->T)))
    return fail(ctx, STRP_EINVAL, "verify_draft: ldt must be a multiple of 8 and not below T + n_seq, ldd of 8 and not below T");
  if (!ptr16(in->target) || (in->T > 0 && !ptr16(in->draft))) return fail(ctx, STRP_EINVAL, "verify_draft: target or draft not 16-byte aligned");
  if (!ctx->ws) return fail(ctx, STRP_ENOMEM, "verify_draft: no workspace set");
  const VerifyPlan q = plan_verify(in->V, in->T, in->n_seq, in->dtype);
  Arena arena(ctx);
  STRP_TAKE(ctx, arena, mass, Mass, (size_t)(2 * in->T + in->n_seq) * q.slices);
  STRP_TAKE(ctx, arena, chosen, Chosen, in->n_seq);
  STRP_TAKE(ctx, arena, sums, double, (size_t)in->n_seq * q.parts * 2);
  OnDevice on(ctx);
  if (!on.ok()) return fail(ctx, STRP_EHIP, "verify_draft: device %d cannot be made current", ctx->device);
  const double cells = (double)in->V * (2.0 * in->T + in->n_seq);
  ProfScope ps(ctx, "verify_draft", 3.0 * cells, bytes_of(in->dtype) * cells);
  const VerifyP p{in->target, in->draft, in->draft_id, in->u, in->u_next, in->draft_start, in->accepted, in->next_id, in->V, in->n_seq, (int)in->T, (int)in->T + in->n_seq,
                  in->ldt, in->ldd, 1.0 / in->temperature, q.ct, q.groups_t, q.slices, q.rows, mass, q.parts, q.part_rows, chosen, sums};
  if (in->dtype == STRP_BF16) launch_verify<__bf16>(ctx, p, q);
  else launch_verify<float>(ctx, p, q);
  STRP_HIP(ctx, hipGetLastError());
  return STRP_OK;
}

}  // extern "C"
