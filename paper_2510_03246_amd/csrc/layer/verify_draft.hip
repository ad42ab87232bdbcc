// Drafted tokens against the target's probabilities, and the token that follows them.
//
//   keep x where u q(x) < p(x);  then the lowest v with sum_{w <= v} r(w) > u' sum r,  r = max(p - q, 0) or p,
// with p and q the softmax of two columns of logits [V x tokens].  What is asked is an index into 10^5 sums, of which some lie within 10^-7 of each other:
// 32 bits would answer beside it once in a few hundred times, so exponentials and sums are of 64.
//
// Four kernels: sums of exponentials over slices of every column (all that is read once; 256 sequences of 4 tokens, 50000 entries of bf16: 87 of 132 us, the vector unit busy 83 % of
// them where memory needs 45); the first token of every sequence that is not kept;
// the sums of r over parts of the vocabulary; the part that holds the answer, entry by entry.
#include "layer_ops.h"

#include <type_traits>

namespace strp {

constexpr int SLICES = 256, PARTS = 256;   // at most: a lane has four of either

// e^y to 2^-43 of itself, for y from -705 to 600, in units of ln 2 / 32: y = 32 k + j + r with |r| <= 1/2, so that e^y = 2^k 2^(j/32) 2^(r/32): a table of 32 in LDS, which 64 banks
// give to any lanes at once, and a polynomial of the fourth degree (the series to r^5 with that power taken for the nearest lower ones on the interval, a Chebyshev polynomial less).
// 10 instructions in 64 bits, 18 an entry in all (verify_256 132 us; without the table and to r^12 22 instructions, and 445 us before the other steps too).
constexpr double LN2 = 0.69314718055994530942, UNITS = 32.0 / LN2;      // of ln 2 / 32 in one
constexpr double LOWEST = -700.0 * UNITS;
struct ExpTable { double of[32]; };
constexpr ExpTable exp_table() {           // 2^(j/32), j < 32, by the series of e^x on [0, ln 2)
  ExpTable t{};
  for (int j = 0; j < 32; ++j) {
    double s = 1.0;
    for (int k = 22; k > 0; --k) s = 1.0 + s * (j / UNITS) / k;
    t.of[j] = s;
  }
  return t;
}
__device__ const ExpTable exp_values = exp_table();
__device__ __forceinline__ void fill_table(double* table) {
  if (threadIdx.x < 32) table[threadIdx.x] = __builtin_bit_cast(double, __builtin_bit_cast(unsigned long long, exp_values.of[threadIdx.x]) - ((unsigned long long)threadIdx.x << 47));
  __syncthreads();
}
struct Exp {
  const double* table;
  __device__ __forceinline__ double near(double y) const {          // y in units
    constexpr double ROUND = 6755399441055744.0;                    // 1.5 2^52: what is added to it is rounded to whole numbers, which its lower bits then have
    constexpr double L = 1.0 / UNITS, A = 0.5 * L, C1 = L * (1.0 - 5.0 * A * A * A * A / 1920.0), C2 = L * L / 2.0, C3 = L * L * L * (1.0 / 6.0 + 20.0 * A * A / 1920.0), C4 = L * L * L * L / 24.0;
    const double t = y + ROUND, r = y - (t - ROUND);
    double p = __builtin_fma(r, C4, C3);
    p = __builtin_fma(p, r, C2);
    p = __builtin_fma(p, r, C1) * r;
    const unsigned i = (unsigned)__builtin_bit_cast(unsigned long long, t);
    // k and j, whole, into the exponent and behind it: the table has j taken off there
    const uint2 of = ((const uint2*)table)[i & 31];
    unsigned high = of.y + (i << 15);
    asm("" : "+v"(high));                  // (or it becomes an addition of 64 bits, three instructions)
    const double b = __builtin_bit_cast(double, (unsigned long long)high << 32 | of.x);
    return __builtin_fma(b, p, b);
  }
  // 0 where y is below -700 or NaN
  __device__ __forceinline__ double of_units(double y) const { return y >= LOWEST ? near(y) : 0.0; }
  __device__ __forceinline__ double operator()(double y) const { return of_units(y * UNITS); }
};

// Sum of e^((x - ref) / temperature) over some entries.  ref is one of them and no more than 500 temperatures below any: with 64 bits it need not be the largest.
// most: the largest, NaN where there is one.
struct __attribute__((aligned(16))) Mass {
  double sum;
  float ref, most;
};

// the column of p, that of q (-1: none), and what makes probabilities of exponentials; bad: no answer
struct Chosen { int col_t, col_d, bad, pad; double ref_t, inv_t, ref_d, inv_d; };

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
  Chosen* chosen;                          // [n_seq]
  double* sums;                            // [n_seq][parts][2] of r and of p
};

// An exponent is x scale - from with from = ref scale, rounded: one instruction, but what that rounding took stays in every exponent, ref's own among them, and grows with ref / temperature.
// It is one number a reference, so the sum by it is put right at its end (otherwise 10^-9 of it at logits of 20 and a temperature of 10^-6, 10^-3 at 10^-12, and anything at 10^-16; the correction costs verify_64 1.3 us of 55, verify_256 1.6 of 132).
// From references of FAR units on differences come first: what is left would outgrow the exponents, and neighbouring logits are 2^21 units apart.
constexpr double FAR = 35184372088832.0;   // 2^45
__device__ __forceinline__ double left_over(float ref, double from, double scale) { return fabs(from) < FAR ? __builtin_fma((double)ref, scale, -from) : 0.0; }

template <typename E>
__global__ __launch_bounds__(256) void verify_sums_kernel(const VerifyP p) {
  constexpr int VEC = 16 / sizeof(E), UN = 2;
  __shared__ double table[32];
  __shared__ double sSum[4][8][VEC];
  __shared__ float sRef[4][8][VEC], sMost[4][8][VEC];
  fill_table(table);
  const Exp ex{table};
  const bool of_draft = (int)blockIdx.x >= p.groups_t;
  const int c = threadIdx.x % p.ct, r = threadIdx.x / p.ct, rl = 256 / p.ct, wave = threadIdx.x >> 6;
  const long long t0 = ((long long)((int)blockIdx.x - (of_draft ? p.groups_t : 0)) * p.ct + c) * VEC, ld = of_draft ? p.ldd : p.ldt;
  const int n = of_draft ? p.T : p.columns, v0 = (int)blockIdx.y * p.rows, v1 = min(v0 + p.rows, p.V);
  double sum[VEC], from[VEC];              // from: ref / temperature, in the units of Exp
  float ref[VEC], most[VEC], high[VEC];    // high: what ref may not stay behind
  bool apart = false;                      // some reference is FAR
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    sum[e] = from[e] = 0.0;
    ref[e] = most[e] = high[e] = -INFINITY;
  }
  // half of what ref may stay behind: the sum of both in 32 bits, rounded upwards from half a step of theirs on, is at most twice as far (by 500 neighbours of 64 at a temperature of
  // 10^-8, 763 apart, were taken for less, and the larger lost)
  const float reach = (float)(250.0 / p.inv);
  const double scale = p.inv * UNITS;
  if (t0 < n) {
    const E* x = (const E*)(of_draft ? p.draft : p.target) + t0;
    struct Rows { uintx4 x[UN]; };
    // rows from `at` on, rl apart, no further than the slice's last: asked for while those before them are worked on
    const E* final_row = x + (long long)(v1 - 1) * ld;
    auto ask = [&](const E* at) {
      Rows rows;
#pragma unroll
      for (int k = 0; k < UN; ++k) {
        const E* from = at + (long long)(k * rl) * ld;
        rows.x[k] = *(const uintx4*)(from < final_row ? from : final_row);
      }
      return rows;
    };
    auto take = [&](auto count, const Rows& rows) {
      constexpr int N = decltype(count)::value;
      float f[N][VEC];
#pragma unroll
      for (int k = 0; k < N; ++k)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const unsigned w = rows.x[k][e * sizeof(E) / 4];
          f[k][e] = __builtin_bit_cast(float, sizeof(E) == 4 ? w : e % 2 ? w & 0xffff0000u : w << 16);
        }
      bool far = false;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        float m = f[0][e];
#pragma unroll
        for (int k = 1; k < N; ++k) m = __builtin_elementwise_maximum(m, f[k][e]);
        most[e] = __builtin_elementwise_maximum(most[e], m);
        far = far || most[e] > high[e];
      }
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(far) != 0, 0)) {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (most[e] > high[e]) {
            const double to = (double)most[e] * scale;
            sum[e] *= ref[e] == -INFINITY ? 0.0 : ex.of_units(((double)ref[e] - (double)most[e]) * scale - left_over(ref[e], from[e], scale) + left_over(most[e], to, scale));
            ref[e] = most[e];
            high[e] = ref[e] + reach;
            from[e] = to;
            apart = apart || !(fabs(to) < FAR);
          }
      }
      // (the lower bound, for -inf and NaN too: e^-700 is nothing beside ref's own share)
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(apart) != 0, 0)) {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
#pragma unroll 1
          for (int k = 0; k < N; ++k) {
            const double y = fabs(from[e]) < FAR ? __builtin_fma((double)f[k][e], scale, -from[e]) : ((double)f[k][e] - (double)ref[e]) * scale;
            sum[e] += ex.near(fmax(y, LOWEST));
          }
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
#pragma unroll
          for (int k = 0; k < N; ++k) sum[e] += ex.near(fmax(__builtin_fma((double)f[k][e], scale, -from[e]), LOWEST));
      }
    };
    int v = v0 + r;
    if (v < v1) {
      const E* at = x + (long long)v * ld;
      const long long step = (long long)(UN * rl) * ld;
      Rows rows = ask(at);
#pragma unroll 1
      for (; v + (UN - 1) * rl < v1; v += UN * rl) {
        at += step;
        const Rows next = ask(at);
        take(std::integral_constant<int, UN>(), rows);
        rows = next;
      }
#pragma unroll 1
      for (; v < v1; v += rl) {
        take(std::integral_constant<int, 1>(), rows);
#pragma unroll
        for (int k = 0; k + 1 < UN; ++k) rows.x[k] = rows.x[k + 1];
      }
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) sum[e] = ref[e] == -INFINITY ? 0.0 : sum[e];
  bool much = false;                       // more than 2^-40 units, which are 2^-45 of a sum (verify_64 54.7 us, 55.3 without the question)
#pragma unroll
  for (int e = 0; e < VEC; ++e) much = much || (sum[e] != 0.0 && fabs(left_over(ref[e], from[e], scale)) > 0x1p-40);
  if (__builtin_amdgcn_ballot_w64(much))
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (sum[e] != 0.0) sum[e] *= ex.near(-left_over(ref[e], from[e], scale));
  // one reference for the slice, and the sums by it: over the wavefront, then the four of them
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    float all = ref[e], top = most[e];
    for (int o = p.ct; o < 64; o <<= 1) {
      all = fmaxf(all, __shfl_xor(all, o, 64));
      top = __builtin_elementwise_maximum(top, __shfl_xor(top, o, 64));
    }
    if (sum[e] != 0.0 && all != ref[e]) sum[e] *= ex(((double)ref[e] - (double)all) * p.inv);
    for (int o = p.ct; o < 64; o <<= 1) sum[e] += __shfl_xor(sum[e], o, 64);
    if ((int)(threadIdx.x & 63) < p.ct) {
      sSum[wave][c][e] = sum[e];
      sRef[wave][c][e] = all;
      sMost[wave][c][e] = top;
    }
  }
  __syncthreads();
  if ((int)threadIdx.x < p.ct * VEC) {
    const int cc = threadIdx.x / VEC, e = threadIdx.x % VEC;
    const long long t = ((long long)((int)blockIdx.x - (of_draft ? p.groups_t : 0)) * p.ct + cc) * VEC + e;
    float all = sRef[0][cc][e], top = sMost[0][cc][e];
#pragma unroll
    for (int w = 1; w < 4; ++w) {
      all = fmaxf(all, sRef[w][cc][e]);
      top = __builtin_elementwise_maximum(top, sMost[w][cc][e]);
    }
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const double x = sSum[w][cc][e];
      if (x != 0.0) s += sRef[w][cc][e] == all ? x : x * ex(((double)sRef[w][cc][e] - (double)all) * p.inv);
    }
    if (t < n) p.mass[(t + (of_draft ? p.columns : 0)) * p.slices + blockIdx.y] = Mass{s, all, top};
  }
}

// All slices of a column, in every lane of the wavefront.
__device__ __forceinline__ Mass whole_column(const VerifyP& p, const Exp& ex, long long column) {
  const int lane = threadIdx.x & 63;
  Mass a[SLICES / 64];
  Mass all = Mass{0.0, -INFINITY, -INFINITY};
#pragma unroll
  for (int i = 0; i < SLICES / 64; ++i) {
    a[i] = Mass{0.0, -INFINITY, -INFINITY};
    if (lane + 64 * i < p.slices) a[i] = p.mass[column * p.slices + lane + 64 * i];
  }
#pragma unroll
  for (int i = 0; i < SLICES / 64; ++i) {
    all.ref = fmaxf(all.ref, a[i].ref);
    all.most = __builtin_elementwise_maximum(all.most, a[i].most);
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    all.ref = fmaxf(all.ref, __shfl_xor(all.ref, o, 64));
    all.most = __builtin_elementwise_maximum(all.most, __shfl_xor(all.most, o, 64));
  }
#pragma unroll
  for (int i = 0; i < SLICES / 64; ++i)
    if (a[i].sum != 0.0) all.sum += a[i].sum * ex(((double)a[i].ref - (double)all.ref) * p.inv);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) all.sum += __shfl_xor(all.sum, o, 64);
  return all;
}

// A workgroup for a sequence, a wavefront for a position.
constexpr int DECIDERS = 8;
template <typename E>
__global__ __launch_bounds__(64 * DECIDERS) void verify_decide_kernel(const VerifyP p) {
  __shared__ double table[32];
  __shared__ int stop[DECIDERS];
  __shared__ Chosen found[DECIDERS];
  fill_table(table);
  const Exp ex{table};
  const int seq = (int)blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const auto begin = [&](int s) { return p.draft_start ? min(max(p.draft_start[s], 0), p.T) : (s ? p.T : 0); };
  const int a = begin(seq), n = max(begin(seq + 1) - a, 0);
  for (int i0 = 0; i0 <= n; i0 += DECIDERS) {
    const int i = i0 + wave;
    if (i <= n) {
      const int ct = min(a + seq + i, p.columns - 1), x = i < n ? p.draft_id[a + i] : 0, at = min(max(x, 0), p.V - 1);
      const float xt = (float)((const E*)p.target)[(long long)at * p.ldt + ct];
      const Mass mt = whole_column(p, ex, ct);
      Chosen c = Chosen{ct, -1, 0, 0, (double)mt.ref, 1.0 / mt.sum, 0.0, 0.0};
      c.bad = !(fabsf(mt.most) < INFINITY);
      bool keep = false;
      if (i < n) {
        const float xd = (float)((const E*)p.draft)[(long long)at * p.ldd + a + i];
        const Mass md = whole_column(p, ex, (long long)p.columns + a + i);
        c.col_d = a + i;
        c.ref_d = md.ref;
        c.inv_d = 1.0 / md.sum;
        c.bad = c.bad || !(fabsf(md.most) < INFINITY);
        if (x == at && !c.bad) keep = (double)p.u[a + i] * (ex(((double)xd - c.ref_d) * p.inv) * c.inv_d) < ex(((double)xt - c.ref_t) * p.inv) * c.inv_t;
      }
      if (lane == 0) {
        stop[wave] = !keep;
        found[wave] = c;
      }
    }
    __syncthreads();
    int at = -1;
    for (int w = DECIDERS - 1; w >= 0; --w)
      if (i0 + w <= n && stop[w]) at = w;
    if (at >= 0) {
      if (threadIdx.x == 0) {
        p.accepted[seq] = i0 + at;
        p.chosen[seq] = found[at];
      }
      break;
    }
    __syncthreads();
  }
}

__device__ __forceinline__ double weight(const Chosen& c, const Exp& ex, float xt, float xd, bool rest, double inv) {
  const double pt = ex(((double)xt - c.ref_t) * inv) * c.inv_t;
  if (!rest) return pt;
  return fmax(pt - ex(((double)xd - c.ref_d) * inv) * c.inv_d, 0.0);
}

// A workgroup has a part of the vocabulary for S sequences: neighbouring lanes are neighbouring sequences, whose columns lie in the same lines of memory.
template <typename E, int S>
__global__ __launch_bounds__(256) void verify_weigh_kernel(const VerifyP p) {
  constexpr int RL = 256 / S, UN = 4;
  __shared__ double table[32];
  __shared__ double sr[4][S], sp[4][S];
  fill_table(table);
  const Exp ex{table};
  const int s = threadIdx.x % S, r0 = threadIdx.x / S, wave = threadIdx.x >> 6, seq = (int)blockIdx.x * S + s, part = (int)blockIdx.y;
  const Chosen c = p.chosen[min(seq, p.n_seq - 1)];
  const int v0 = part * p.part_rows, v1 = min(v0 + p.part_rows, p.V);
  double r = 0.0, q = 0.0;
  if (!c.bad) {
    const E* target = (const E*)p.target + c.col_t;
    const E* draft = (const E*)p.draft + max(c.col_d, 0);
    const bool drafted = c.col_d >= 0;
    for (int v = v0 + r0; v < v1; v += UN * RL) {
      float xt[UN], xd[UN];
#pragma unroll
      for (int k = 0; k < UN; ++k) {
        const long long at = min(v + k * RL, v1 - 1);
        xt[k] = (float)target[at * p.ldt];
        xd[k] = drafted ? (float)draft[at * p.ldd] : 0.0f;
      }
#pragma unroll
      for (int k = 0; k < UN; ++k) {
        const bool in = v + k * RL < v1;
        const double pt = ex(((double)xt[k] - c.ref_t) * p.inv) * c.inv_t;
        q += in ? pt : 0.0;
        if (drafted) r += in ? fmax(pt - ex(((double)xd[k] - c.ref_d) * p.inv) * c.inv_d, 0.0) : 0.0;
      }
    }
  }
#pragma unroll
  for (int o = S; o < 64; o <<= 1) {
    r += __shfl_xor(r, o, 64);
    q += __shfl_xor(q, o, 64);
  }
  if ((int)(threadIdx.x & 63) < S) {
    sr[wave][s] = r;
    sp[wave][s] = q;
  }
  __syncthreads();
  if ((int)threadIdx.x < S && seq < p.n_seq) {
    double* to = p.sums + ((long long)seq * p.parts + part) * 2;
    to[0] = ((sr[0][s] + sr[1][s]) + sr[2][s]) + sr[3][s];
    to[1] = ((sp[0][s] + sp[1][s]) + sp[2][s]) + sp[3][s];
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
  __shared__ double table[32];
  __shared__ double totals[4];
  __shared__ int firsts[4], lasts[4];
  const int seq = (int)blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  fill_table(table);
  const Exp ex{table};
  const Chosen c = p.chosen[seq];
  if (c.bad) {
    if (threadIdx.x == 0) p.next_id[seq] = -1;
    return;
  }
  // every wavefront finds the part for itself
  const double* from = p.sums + (long long)seq * p.parts * 2;
  double r[PARTS / 64], s[PARTS / 64], rs = 0.0, ss = 0.0;      // lane l has the parts 4 l and on
#pragma unroll
  for (int i = 0; i < PARTS / 64; ++i) {
    const int at = PARTS / 64 * lane + i;
    const bool in = at < p.parts;
    r[i] = in && c.col_d >= 0 ? from[2 * at] : 0.0;
    s[i] = in ? from[2 * at + 1] : 0.0;
    rs += r[i];
    ss += s[i];
  }
  const bool rest = __builtin_amdgcn_ballot_w64(rs > 0.0) != 0;
  const double mine = rest ? rs : ss, sum = upto(mine), total = __shfl(sum, 63, 64);
  const float u = p.u_next[seq];
  const double goal = u < 1.0f ? (double)u * total : (double)INFINITY;
  const unsigned long long over = __builtin_amdgcn_ballot_w64(sum > goal && mine > 0.0), some = __builtin_amdgcn_ballot_w64(mine > 0.0);
  const int holder = over ? __builtin_ctzll(over) : some ? 63 - __builtin_clzll(some) : 0;
  // of the holder's parts the first whose sum is over the goal, or the last that has any
  double before = __shfl(sum - mine, holder, 64);
  int part = PARTS / 64 * holder;
  {
    double run = before;
    bool done = false;
#pragma unroll
    for (int i = 0; i < PARTS / 64; ++i) {
      const double x = __shfl(rest ? r[i] : s[i], holder, 64);
      if (!done && x > 0.0) {
        before = run;
        part = PARTS / 64 * holder + i;
      }
      run += x;
      done = done || (x > 0.0 && run > goal);
    }
  }
  // its entries, 256 at a time
  const int v0 = part * p.part_rows, v1 = min(v0 + p.part_rows, p.V);
  int last = -1;                           // the last entry with r > 0, should rounding leave the sums of the part below the goal
  for (int b = v0; b < v1; b += 256) {
    const int v = b + (int)threadIdx.x;
    double w = 0.0;
    if (v < v1) w = weight(c, ex, (float)((const E*)p.target)[(long long)v * p.ldt + c.col_t], rest ? (float)((const E*)p.draft)[(long long)v * p.ldd + c.col_d] : 0.0f, rest, p.inv);
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

constexpr int WIDEST = 8;                  // 16-byte columns of a workgroup: a line of 128 bytes
struct VerifyPlan {
  int ct, groups_t, groups_d, slices, rows, parts, part_rows;
};
static VerifyPlan plan_verify(int V, long long T, int n_seq, int dtype) {
  VerifyPlan q;
  const long long vec = dtype == STRP_BF16 ? 8 : 4, chunks_t = (T + n_seq + vec - 1) / vec, chunks_d = (T + vec - 1) / vec;
  q.ct = 1;
  while (q.ct < WIDEST && q.ct < chunks_t) q.ct *= 2;
  q.groups_t = (int)((chunks_t + q.ct - 1) / q.ct);
  q.groups_d = (int)((chunks_d + q.ct - 1) / q.ct);
  // as many workgroups as the chip holds at once, three a CU in bf16 and six in fp32 (verify_256 131 us; 1024 workgroups 134, 2048 138), none below one entry a thread
  long long slices = (dtype == STRP_BF16 ? 768 : 1536) / (q.groups_t + q.groups_d);
  if (slices < 1) slices = 1;
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
  const dim3 block(256);
  const unsigned n = (unsigned)p.n_seq;
  hipLaunchKernelGGL((verify_sums_kernel<E>), dim3((unsigned)(q.groups_t + q.groups_d), (unsigned)q.slices), block, 0, ctx->stream, p);
  hipLaunchKernelGGL((verify_decide_kernel<E>), dim3(n), dim3(64 * DECIDERS), 0, ctx->stream, p);
  // neighbouring sequences' columns lie in the same lines of memory, so many a workgroup, as long as the chip is full (64 sequences: 16 a workgroup 17 us, 8 25; 256: 32 42 us, 16 50)
  if (n >= 128) hipLaunchKernelGGL((verify_weigh_kernel<E, 32>), dim3((n + 31) / 32, (unsigned)q.parts), block, 0, ctx->stream, p);
  else if (n >= 8) hipLaunchKernelGGL((verify_weigh_kernel<E, 16>), dim3((n + 15) / 16, (unsigned)q.parts), block, 0, ctx->stream, p);
  else hipLaunchKernelGGL((verify_weigh_kernel<E, 1>), dim3(n, (unsigned)q.parts), block, 0, ctx->stream, p);
  hipLaunchKernelGGL((verify_find_kernel<E>), dim3(n), block, 0, ctx->stream, p);
}

}  // namespace strp

using namespace strp;

extern "C" {

size_t strp_verify_draft_workspace_bytes(int32_t V, int64_t T, int32_t n_seq) {
  if (V <= 0 || V > (1 << 30) || T < 0 || T > (1 << 20) || n_seq <= 0 || n_seq > 65536) return 0;
  // What plan_verify makes of these sizes or of smaller ones, in either type: more slices than one only where their workgroups, of up to 128 bytes of columns, are no more than 768 (fp32:
  // 1536) in all.  (256 for every column asked for 9.1 GB at 2^20 drafted tokens of 65536 sequences, which take 0.31.)
  const size_t columns = 2 * (size_t)T + n_seq, at_once = (size_t)768 * WIDEST * 8, most = (size_t)(V + 256 / WIDEST - 1) / (256 / WIDEST);
  const size_t each = columns * (most < SLICES ? most : SLICES), all = columns > at_once ? columns : at_once;
  const size_t parts = (size_t)(V + 255) / 256;
  // (a workspace has 4 KB at least)
  return 4096 + up256((each < all ? each : all) * sizeof(Mass)) + up256((size_t)n_seq * sizeof(Chosen)) + up256((size_t)n_seq * (parts < PARTS ? parts : PARTS) * 16);
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
