// Keys and values of new tokens into the pages of a cache, keys and queries turned by their positions.
//
//   (x, y) -> (x cos a - y sin a, y cos a + x sin a),  a = position * inv_freq[j]
// in 64 bits: far positions lose all of a 32-bit angle, and what 4 bits hold jumps where a value crosses the middle of two steps.
#include "paged_cache.h"

#include <type_traits>

namespace strp {

struct AppendP {
  Pages c;
  void* cK;
  void* cV;
  float* sK;
  float* sV;
  const void* K;
  const void* V;
  const void* Q;
  void* Qr;
  const float* inv_freq;
  int heads, rot, pairs, items, per;      // items: heads of K, of V and of Q, `per` of them a workgroup
  long long ldk, ldv, ldq, ldqr;
};

// sin and cos of a in 64 bits: a less a multiple of pi/2 in three parts (each product with its part is exact within fma), then the
// series of sine and cosine on [-pi/4, pi/4], whose first left-out terms are below 1e-19.
__device__ __forceinline__ void sin_cos(double a, double& s, double& c) {
  const double n = __builtin_rint(a * 0.63661977236758134308);
  double r = __builtin_fma(-n, 1.5707963267948965580e+00, a);
  r = __builtin_fma(-n, 6.1232339957367660359e-17, r);
  r = __builtin_fma(-n, -1.4973849048591833166e-33, r);
  const double z = r * r;
  double p = 1.0 / 355687428096000.0, q = -1.0 / 6402373705728000.0;
  p = __builtin_fma(p, z, -1.0 / 1307674368000.0);
  p = __builtin_fma(p, z, 1.0 / 6227020800.0);
  p = __builtin_fma(p, z, -1.0 / 39916800.0);
  p = __builtin_fma(p, z, 1.0 / 362880.0);
  p = __builtin_fma(p, z, -1.0 / 5040.0);
  p = __builtin_fma(p, z, 1.0 / 120.0);
  p = __builtin_fma(p, z, -1.0 / 6.0);
  const double sr = __builtin_fma(p * z, r, r);
  q = __builtin_fma(q, z, 1.0 / 20922789888000.0);
  q = __builtin_fma(q, z, -1.0 / 87178291200.0);
  q = __builtin_fma(q, z, 1.0 / 479001600.0);
  q = __builtin_fma(q, z, -1.0 / 3628800.0);
  q = __builtin_fma(q, z, 1.0 / 40320.0);
  q = __builtin_fma(q, z, -1.0 / 720.0);
  q = __builtin_fma(q, z, 1.0 / 24.0);
  q = __builtin_fma(q, z, -0.5);
  const double cr = __builtin_fma(q, z, 1.0);
  const double quarter = n - 4.0 * __builtin_floor(n * 0.25);      // 0, 1, 2 or 3
  const bool odd = quarter == 1.0 || quarter == 3.0;
  s = odd ? cr : sr;
  c = odd ? sr : cr;
  s = quarter >= 2.0 ? -s : s;
  c = quarter == 1.0 || quarter == 2.0 ? -c : c;
}

constexpr int MAXS = 1024;                 // sequences whose offsets a workgroup keeps in LDS

// Positions of TT tokens from t_first on (-1: in no sequence) and their rows of the cache's first head (-1: not stored).
template <int TT, int THREADS>
__device__ __forceinline__ void find_places(const AppendP& p, int t_first, int (&starts)[MAXS + 1], int (&sPos)[TT], long long (&sSlot)[TT]) {
  const int tid = threadIdx.x;
  const bool held = p.c.n_seq <= MAXS;
  if (held && p.c.seq_start) {
    for (int i = tid; i <= p.c.n_seq; i += THREADS) starts[i] = p.c.seq_start[i];
  }
  __syncthreads();
  if (tid < TT) {
    int pos = -1;
    long long slot = -1;
    const int t0 = t_first + tid;
    if (t0 < p.c.T) {
      int s = 0, begin = 0;
      bool in = true;
      if (p.c.seq_start) {
        int a = -1, b = p.c.n_seq + 1;     // seq_start[a] <= t < seq_start[b]
        while (b - a > 1) {
          const int m = (a + b) >> 1;
          if ((held ? starts[m] : p.c.seq_start[m]) <= t0) a = m;
          else b = m;
        }
        in = a >= 0 && a < p.c.n_seq;
        s = in ? a : 0;
        begin = max(held ? starts[s] : p.c.seq_start[s], 0);
      }
      if (in) {
        pos = seq_past(p.c, s) + t0 - begin;
        const int given = p.c.past[s];
        if (given >= 0 && given <= p.c.cap && pos >= 0 && pos < p.c.cap) {
          const int page = p.c.table[(long long)s * p.c.ld_table + (pos >> p.c.page_log2)];
          if (page >= 0 && page < p.c.pages) slot = ((long long)page * p.c.kv_heads << p.c.page_log2) + (pos & ((1 << p.c.page_log2) - 1));
        }
      }
    }
    sPos[tid] = pos;
    sSlot[tid] = slot;
  }
  __syncthreads();
}

// The heads in `tile` into the rows of their tokens: a row by DHP / 8 neighbouring threads, eight channels each.
template <typename E, bool Q4, int TT, int DHP, int THREADS>
__device__ __forceinline__ void store_rows(const AppendP& p, bool isK, int h, const float (&tile)[TT][DHP + 1], const long long (&sSlot)[TT]) {
  const int tid = threadIdx.x, dh = p.c.dh;
  constexpr int PER = DHP / 8;
  void* pool = isK ? p.cK : p.cV;
  float* scales = isK ? p.sK : p.sV;
#pragma unroll
  for (int at = tid; at < TT * PER; at += THREADS) {
    const int row = at / PER, ch = (at % PER) * 8;
    const long long slot = sSlot[row];
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = ch < dh ? tile[row][ch + e] : tile[row][e];
    if constexpr (Q4) {
      float lo = v[0], hi = v[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) {
        lo = __builtin_elementwise_minimum(lo, v[e]);      // NaN stays NaN
        hi = __builtin_elementwise_maximum(hi, v[e]);
      }
#pragma unroll
      for (int o = PER / 2; o > 0; o >>= 1) {
        lo = __builtin_elementwise_minimum(lo, __shfl_xor(lo, o, 64));
        hi = __builtin_elementwise_maximum(hi, __shfl_xor(hi, o, 64));
      }
      // what is not finite, or too far apart: NaN, since a score of minus infinity would hide a key of infinity
      const bool fine = fabsf(hi - lo) < INFINITY && fabsf(lo) < INFINITY;
      const float step = fine ? (hi - lo) / 15.0f : __builtin_nanf("");
      lo = fine ? lo : __builtin_nanf("");
      unsigned w = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float n = step > 0.0f ? __builtin_rintf((v[e] - lo) / step) : 0.0f;
        w |= (unsigned)fminf(fmaxf(n, 0.0f), 15.0f) << (4 * e);
      }
      if (slot >= 0 && ch < dh) {
        const long long r = slot + ((long long)h << p.c.page_log2);
        *(unsigned*)((char*)pool + r * (dh / 2) + ch / 2) = w;
        if (ch == 0) *(float2*)(scales + 2 * r) = float2{lo, step};
      }
    } else if (slot >= 0 && ch < dh) {
      const long long r = slot + ((long long)h << p.c.page_log2);
      E* out = (E*)pool + r * dh + ch;
      if constexpr (sizeof(E) == 2) {
        store_floats<8>(out, v);
      } else {
        const float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
        store_floats<4>(out, a);
        store_floats<4>(out + 4, b);
      }
    }
  }
}

// Few tokens: a workgroup has TT of them and `per` heads of K, V or Q; a thread has a token and every (threads / TT)th pair of channels, for which it works sine and cosine out
// once.  Queries go from row to row as they lie.  Keys and values are turned round through LDS into rows of the cache.
template <typename E, bool Q4, int TT, int DHP>
__global__ __launch_bounds__(256) void append_few_kernel(const AppendP p) {
  constexpr int THREADS = 256, NG = THREADS / TT, NP = (DHP / 2 + NG - 1) / NG;
  __shared__ float tile[TT][DHP + 1];
  __shared__ int starts[MAXS + 1];
  __shared__ int sPos[TT];
  __shared__ long long sSlot[TT];          // row of the cache's first head, -1: not stored
  const int tid = threadIdx.x, tok = tid % TT, grp = tid / TT, t = (int)blockIdx.x * TT + tok;
  const int dh = p.c.dh, half = p.rot / 2;
  const int first = (int)blockIdx.y * p.per, last = min(first + p.per, p.items);

  find_places<TT, THREADS>(p, (int)blockIdx.x * TT, starts, sPos, sSlot);
  const int pos = sPos[tok];

  double cosv[NP], sinv[NP];
  // values are not turned: where the workgroup has nothing else there is nothing to work out
  const bool only_v = first >= p.c.kv_heads && last <= 2 * p.c.kv_heads;
  if (!only_v)
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int j = grp + NG * i;
      cosv[i] = 1.0;
      sinv[i] = 0.0;
      if (j < half) sin_cos((double)pos * (double)p.inv_freq[j], sinv[i], cosv[i]);
    }

  for (int item = first; item < last; ++item) {
    const bool isK = item < p.c.kv_heads, isV = !isK && item < 2 * p.c.kv_heads;
    const int h = isK ? item : item - p.c.kv_heads * (isV ? 1 : 2);
    const long long ld = isK ? p.ldk : isV ? p.ldv : p.ldq;
    const E* src = (const E*)(isK ? p.K : isV ? p.V : p.Q) + (long long)h * dh * ld + t;
    E* dst = (E*)p.Qr + (long long)h * dh * p.ldqr + t;
    float x[NP], y[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int j = grp + NG * i;
      const bool turned = j < half, split = turned && !p.pairs;
      const int c0 = split ? j : 2 * j, c1 = split ? j + half : 2 * j + 1;
      const bool in = 2 * j < dh && t < p.c.T;
      x[i] = y[i] = 0.0f;
      if (in) {
        x[i] = (float)src[c0 * ld];
        y[i] = (float)src[c1 * ld];
      }
    }
    if (!isV)
#pragma unroll
      for (int i = 0; i < NP; ++i)
        if (grp + NG * i < half) {
          const double a = x[i], b = y[i];
          x[i] = (float)(a * cosv[i] - b * sinv[i]);
          y[i] = (float)(b * cosv[i] + a * sinv[i]);
        }
    if (!isK && !isV) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int j = grp + NG * i;
        const bool split = j < half && !p.pairs;
        const int c0 = split ? j : 2 * j, c1 = split ? j + half : 2 * j + 1;
        if (2 * j < dh && pos >= 0) {
          dst[c0 * p.ldqr] = (E)x[i];
          dst[c1 * p.ldqr] = (E)y[i];
        }
      }
      continue;
    }
    __syncthreads();                       // the tile of the head before has been read
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int j = grp + NG * i;
      const bool split = j < half && !p.pairs;
      const int c0 = split ? j : 2 * j, c1 = split ? j + half : 2 * j + 1;
      if (2 * j < dh) {
        tile[tok][c0] = x[i];
        tile[tok][c1] = y[i];
      }
    }
    __syncthreads();
    store_rows<E, Q4, TT, DHP, THREADS>(p, isK, h, tile, sSlot);
  }
}

// Many tokens, 64 a workgroup: a thread has four neighbours of them, 8 bytes (fp32: 16) of a channel, and two pairs of channels of each head, the next head's asked for while this one is
// turned and stored.  Bound by memory: eight prompts of 2048 tokens, 32 heads of 64, 88 us, 4.6 TB/s (a token and 2 bytes a thread: 197).
template <typename E, bool Q4, int DHP>
__global__ __launch_bounds__(4 * DHP) void append_many_kernel(const AppendP p) {
  constexpr int TT = 64, THREADS = 4 * DHP, NG = THREADS / 16;
  typedef E vec __attribute__((ext_vector_type(4)));
  __shared__ float tile[TT][DHP + 1];
  __shared__ int starts[MAXS + 1];
  __shared__ int sPos[TT];
  __shared__ long long sSlot[TT];
  const int tid = threadIdx.x, tok = 4 * (tid & 15), grp = tid >> 4, t = (int)blockIdx.x * TT + tok;
  const int dh = p.c.dh, half = p.rot / 2;
  const int first = (int)blockIdx.y * p.per, last = min(first + p.per, p.items);

  int c0[2], c1[2];                        // the thread's pairs of channels
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int j = grp + NG * i;
    const bool split = j < half && !p.pairs;
    c0[i] = split ? j : 2 * j;
    c1[i] = split ? j + half : 2 * j + 1;
  }
  const bool in = t < p.c.T;
  struct Item { vec x[2], y[2]; };
  auto ask = [&](int item) {
    const bool isK = item < p.c.kv_heads, isV = !isK && item < 2 * p.c.kv_heads;
    const int h = isK ? item : item - p.c.kv_heads * (isV ? 1 : 2);
    const long long ld = isK ? p.ldk : isV ? p.ldv : p.ldq;
    const E* src = (const E*)(isK ? p.K : isV ? p.V : p.Q) + (long long)h * dh * ld + t;
    Item r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      r.x[i] = r.y[i] = vec{(E)0.0f, (E)0.0f, (E)0.0f, (E)0.0f};
      if (in && 2 * (grp + NG * i) < dh) {       // (rows are whole eights of tokens: nothing behind a row is read)
        r.x[i] = *(const vec*)(src + c0[i] * ld);
        r.y[i] = *(const vec*)(src + c1[i] * ld);
      }
    }
    return r;
  };
  Item next = ask(first);
  find_places<TT, THREADS>(p, (int)blockIdx.x * TT, starts, sPos, sSlot);
  int pos[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) pos[k] = sPos[tok + k];

  double cosv[2][4], sinv[2][4];
  // values are not turned: where the workgroup has nothing else there is nothing to work out
  const bool only_v = first >= p.c.kv_heads && last <= 2 * p.c.kv_heads;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      cosv[i][k] = 1.0;
      sinv[i][k] = 0.0;
    }
  if (!only_v)
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (grp + NG * i < half) {
        const double f = (double)p.inv_freq[grp + NG * i];
#pragma unroll
        for (int k = 0; k < 4; ++k) sin_cos((double)pos[k] * f, sinv[i][k], cosv[i][k]);
      }

  for (int item = first; item < last; ++item) {
    const bool isK = item < p.c.kv_heads, isV = !isK && item < 2 * p.c.kv_heads;
    const int h = isK ? item : item - p.c.kv_heads * (isV ? 1 : 2);
    const Item now = next;
    if (item + 1 < last) next = ask(item + 1);
    float x[2][4], y[2][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[i][k] = (float)now.x[i][k];
        y[i][k] = (float)now.y[i][k];
        if (!isV && grp + NG * i < half) {
          const double a = x[i][k], b = y[i][k];
          x[i][k] = (float)(a * cosv[i][k] - b * sinv[i][k]);
          y[i][k] = (float)(b * cosv[i][k] + a * sinv[i][k]);
        }
      }
    if (!isK && !isV) {
      E* dst = (E*)p.Qr + (long long)h * dh * p.ldqr + t;
      const bool all = in && pos[0] >= 0 && pos[1] >= 0 && pos[2] >= 0 && pos[3] >= 0;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (2 * (grp + NG * i) < dh) {
          if (all) {
            store_floats<4>(dst + c0[i] * p.ldqr, x[i]);
            store_floats<4>(dst + c1[i] * p.ldqr, y[i]);
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (pos[k] >= 0) {
                dst[c0[i] * p.ldqr + k] = (E)x[i][k];
                dst[c1[i] * p.ldqr + k] = (E)y[i][k];
              }
          }
        }
      continue;
    }
    __syncthreads();                       // the tile of the head before has been read
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (2 * (grp + NG * i) < dh)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          tile[tok + k][c0[i]] = x[i][k];
          tile[tok + k][c1[i]] = y[i][k];
        }
    __syncthreads();
    store_rows<E, Q4, TT, DHP, THREADS>(p, isK, h, tile, sSlot);
  }
}

constexpr int FEW = 8, MANY = 64;          // tokens a workgroup
template <typename E, bool Q4>
static void launch_append(strp_ctx* ctx, AppendP p) {
  const bool few = p.c.T <= 64;
  const int tiles = few ? (p.c.T + FEW - 1) / FEW : (p.c.T + MANY - 1) / MANY;
  p.items = 2 * p.c.kv_heads + (p.Q ? p.heads : 0);
  // Sine and cosine are worked out once for the heads of a workgroup: as many heads, up to eight, as leave the chip what it holds at once (with 16 heads of 64 a workgroup 94 us, with 8 or 4
  // 88; 3523 tokens, 48 heads of 128, 4 bits: 512 workgroups 30.1 us, 768 28.6, 1024 29.1).
  const long long wgs = (long long)tiles * p.items;
  const long long resident = few ? 1024 : p.c.dh > 64 ? 768 : 1024, per = (wgs + resident - 1) / resident;
  p.per = (int)(per < 8 ? per : 8);
  const dim3 grid((unsigned)tiles, (unsigned)((p.items + p.per - 1) / p.per));
  const auto go = [&](auto width) {
    constexpr int DHP = decltype(width)::value;
    if (few) hipLaunchKernelGGL((append_few_kernel<E, Q4, FEW, DHP>), grid, dim3(256), 0, ctx->stream, p);
    else hipLaunchKernelGGL((append_many_kernel<E, Q4, DHP>), grid, dim3(4 * DHP), 0, ctx->stream, p);
  };
  if (p.c.dh <= 32) go(std::integral_constant<int, 32>());
  else if (p.c.dh <= 64) go(std::integral_constant<int, 64>());
  else go(std::integral_constant<int, 128>());
}

}  // namespace strp

using namespace strp;

extern "C" strp_status strp_cache_append(strp_ctx* ctx, const strp_cache_append_in* in) {
  if (!ctx) return STRP_EINVAL;
  if (!in || !in->K || !in->V) return fail(ctx, STRP_EINVAL, "cache_append: null K or V");
  if (const char* e = cache_error(in->cache, in->dtype, in->Q ? in->heads : 1, in->T)) return fail(ctx, STRP_EINVAL, "cache_append: %s", e);
  if ((in->Q == nullptr) != (in->Qr == nullptr)) return fail(ctx, STRP_EINVAL, "cache_append: Q and Qr belong together");
  if (in->rot < 0 || in->rot > in->cache.d_head || in->rot % 2) return fail(ctx, STRP_EINVAL, "cache_append: rot must be even, from 0 to d_head");
  if (in->rot && !in->inv_freq) return fail(ctx, STRP_EINVAL, "cache_append: rot > 0 needs inv_freq");
  if (!token_ld(in->ldk, in->T) || !token_ld(in->ldv, in->T) || (in->Q && (!token_ld(in->ldq, in->T) || !token_ld(in->ldqr, in->T))))
    return fail(ctx, STRP_EINVAL, "cache_append: leading dimensions must be multiples of 8 and not below T");
  if (in->Q && in->Q == in->Qr && in->ldq != in->ldqr) return fail(ctx, STRP_EINVAL, "cache_append: Qr may be Q itself with the same ld");
  if (!ptr16(in->K) || !ptr16(in->V) || !ptr16(in->Q) || !ptr16(in->Qr)) return fail(ctx, STRP_EINVAL, "cache_append: K, V, Q or Qr not 16-byte aligned");
  OnDevice on(ctx);
  if (!on.ok()) return fail(ctx, STRP_EHIP, "cache_append: device %d cannot be made current", ctx->device);
  const strp_cache& c = in->cache;
  const AppendP p{pages_of(c, in->T), c.K, c.V, c.K_scale, c.V_scale, in->K, in->V, in->Q, in->Qr, in->inv_freq, in->heads, in->rot, in->pairs != 0, 0, 1,
                  in->ldk, in->ldv, in->ldq, in->ldqr};
  const bool q4 = c.format == STRP_CACHE_Q4;
  const double b = (double)bytes_of(in->dtype), row = q4 ? 0.5 * c.d_head + 8.0 : b * c.d_head, T = (double)in->T;
  const double heads = in->Q ? in->heads : 0;
  ProfScope ps(ctx, "cache_append", 3.0 * T * in->rot * (heads + c.kv_heads), T * (2.0 * b * heads * c.d_head + 2.0 * c.kv_heads * (b * c.d_head + row)));
  if (in->dtype == STRP_BF16) {
    if (q4) launch_append<__bf16, true>(ctx, p);
    else launch_append<__bf16, false>(ctx, p);
  } else {
    if (q4) launch_append<float, true>(ctx, p);
    else launch_append<float, false>(ctx, p);
  }
  STRP_HIP(ctx, hipGetLastError());
  return STRP_OK;
}
