// Attention of new tokens over a paged cache, few rows at a time.
//
//   c = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q . k_j - m),  j = 0 .. position of the token.
// A row is a head at a token; the rows that share keys (the heads of a group, the new tokens of a sequence) are taken 16 at a time.  The work is cut into units, a
// tile of rows by 128 (fp32: 64) keys, numbered sequence by sequence, and every workgroup gets as many of them as any other, one after the other: so a long sequence
// beside short ones, or one alone, fills the chip as well as many alike.  The lengths are in device memory, so every workgroup works its share out
// for itself.  What it does not finish it leaves as (maximum, sum, weighted sum) in the workspace, and a second kernel puts such parts together in their order.
// Bound by memory (64 sequences of 2048 keys, 32 heads of 128 on 8, bf16: 103 us, 5.2 TB/s, a large copy's rate); 4 bits: 3.9 TB/s, the vector unit busy half of the time.
#include "cache_attention.h"
#include "cache_wide.h"

#include <type_traits>

namespace strp {

// One tile of the cache's keys or values as a lane has it.  Keys: lane (key l % 16, quarter l / 16 of a step of the contraction).  Values: channels W (l % 16) .. + W of
// the keys 4 (l / 16) .. + 4, which is where the probabilities of the scores' registers are.
//   E: type of the activations; Q4; W: channels of a value's lane, 16 W >= d_head
template <typename E, bool Q4, int W>
struct Tile;

template <int W>
struct Tile<__bf16, false, W> {
  static constexpr int NC = W / 2;
  typedef uintx4 Key;
  Key k[NC];
  unsigned v[4][W / 2];
};
template <int W>
struct Tile<float, false, W> {
  static constexpr int NC = W;
  typedef floatx4 Key;
  Key k[NC];
  float v[4][W];
};
template <typename E, int W>
struct TileQ4 {
  static constexpr int NC = W / 2;
  unsigned k[NC];
  unsigned v[4];
  floatx4 ks[2], vs[2];
};
template <int W>
struct Tile<__bf16, true, W> : TileQ4<__bf16, W> {};
template <int W>
struct Tile<float, true, W> : TileQ4<float, W> {};

template <int W>
struct RowsLds {
  static constexpr int PITCH = 16 * W + 4;
  float o[4][ROWS][PITCH];
};

template <typename E, bool Q4, int W, bool SPLIT>
__device__ __forceinline__ void rows_share(const RowsP& p, const Heads& heads, unsigned char* smem, unsigned block) {
  constexpr bool BF = sizeof(E) == 2;
  typedef Tile<E, Q4, W> TileT;
  constexpr int NC = TileT::NC, DH = 16 * W;
  constexpr int NT = BF || Q4 ? 2 : 1, KW = 16 * NT, UNIT = 4 * KW;      // tiles and keys of a wavefront in a unit, keys of a unit
  // units that a tile counts beyond its keys' (64 sequences of 0 to 4000 keys, bf16: none 143 us, 1 134, 2 120, 4 121; the fp32 case 2 48 us, 1 46)
  constexpr int EXTRA = BF ? 2 : 1;
  auto& sO = ((RowsLds<W>*)smem)->o;
  __shared__ float sM[4][ROWS], sL[4][ROWS];
  __shared__ long long sOff[ROWS];
  constexpr int HELD = 512;
  __shared__ int sBegin[HELD + 1], sPast[HELD];
  __shared__ __attribute__((aligned(16))) E sQ[ROWS][DH + 8];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n16 = lane & 15, quad = lane >> 4;
  const Pages& c = p.c;
  const int dh = c.dh;
  // neighbours in the work are neighbours on an XCD
  const int worker = (int)(block & 7) * (WORKERS >> 3) + (int)(block >> 3);

  auto tiles_of = [&](int n, int group) { return p.wide && n * group > WIDE_FROM ? 0 : (n * group + ROWS - 1) / ROWS; };      // of the rows that share a key-value head
  auto all_tiles = [&](int n) {            // of a sequence with n new tokens
    if (!heads.first) return c.kv_heads * tiles_of(n, heads.group);
    int sum = 0;
    for (int g = 0; g < c.kv_heads; ++g) sum += tiles_of(n, heads.of(g));
    return sum;
  };
  const bool held = c.n_seq <= HELD;
  if (held) {
    for (int i = tid; i <= c.n_seq; i += 256) {
      sBegin[i] = seq_begin(c, i);
      if (i < c.n_seq) sPast[i] = seq_past(c, i);
    }
    __syncthreads();
  }
  struct Seq { int begin, n, past, units, tiles; };
  auto sequence = [&](int s) {
    Seq q;
    q.begin = held ? sBegin[s] : seq_begin(c, s);
    q.n = max((held ? sBegin[s + 1] : seq_begin(c, s + 1)) - q.begin, 0);
    q.past = held ? sPast[s] : seq_past(c, s);
    q.units = q.n ? (min(q.past + q.n, c.cap) + UNIT - 1) / UNIT + EXTRA : 0;
    q.tiles = q.n ? all_tiles(q.n) : 0;
    return q;
  };
  // this workgroup's units, and the sequence that they begin in
  const int each = (c.n_seq + 63) / 64;
  long long mine = 0;
  for (int i = 0; i < each; ++i)
    if (lane * each + i < c.n_seq) {
      const Seq q = sequence(lane * each + i);
      mine += (long long)q.units * q.tiles;
    }
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long x = __shfl_up(upto, o, 64);
    upto += lane >= o ? x : 0;
  }
  const long long total = uniform(__shfl(upto, 63, 64));
  long long per = (total + WORKERS - 1) / WORKERS;
  per = per < p.least ? p.least : per;
  long long u = worker * per;
  const long long u1 = u + per < total ? u + per : total;
  if (tid == 0) p.parts[worker] = 0;
  if (tid < 2 * ROWS) p.off[(long long)worker * 2 * ROWS + tid] = -1;
  if (u >= u1) return;
  const unsigned long long holds = __builtin_amdgcn_ballot_w64(upto - mine <= u && u < upto);
  const int holder = __builtin_ctzll(holds);
  int s = __builtin_amdgcn_readfirstlane(holder * each);
  long long base = uniform(__shfl(upto - mine, holder, 64));
  auto same = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  auto uniform_sequence = [&] {
    const Seq x = sequence(s);
    return Seq{same(x.begin), same(x.n), same(x.past), same(x.units), same(x.tiles)};
  };
  Seq q = uniform_sequence();
  auto next_sequence = [&] {
    base += (long long)q.units * q.tiles;
    ++s;
    q = uniform_sequence();
  };

  // A segment: units b0 .. b1 of one tile of rows.  The one behind it is known while it is worked on: its first keys and values are on their way before the last ones here are done
  // with, or nothing would be read while the wavefronts join their results (512 sequences of 127 keys, eight segments a workgroup: 87 us, 108 with the queries asked for between segments).
  struct Segment { int s, begin, past, keys, units, kv, rt, group, rows, b0, b1, all; long long last; };      // all: units of the share; last: the tile's last one
  auto segment_at = [&](long long u) {
    while (u >= base + (long long)q.units * q.tiles) next_sequence();
    Segment g{s, q.begin, q.past, min(q.past + q.n, c.cap), q.units - EXTRA, 0, 0, 0, 0, 0, 0, 0, 0};
    const long long rel = u - base;
    const int row_tile = (int)(rel / q.units), from = (int)(rel - (long long)row_tile * q.units), to = (long long)q.units - from < u1 - u ? q.units : from + (int)(u1 - u);
    g.b0 = max(from - EXTRA, 0);
    g.b1 = max(to - EXTRA, 0);
    g.all = to - from;
    g.last = u - from + q.units - 1;
    g.rt = row_tile;
    if (!heads.first) {
      const int per_kv = tiles_of(q.n, heads.group);
      g.kv = row_tile / per_kv;
      g.rt = row_tile - g.kv * per_kv;
      g.group = heads.group;
    } else {
      for (; g.kv < c.kv_heads - 1; ++g.kv) {
        const int t = tiles_of(q.n, same(heads.of(g.kv)));
        if (g.rt < t) break;
        g.rt -= t;
      }
      g.group = same(heads.of(g.kv));
    }
    g.rows = min(ROWS, q.n * g.group - g.rt * ROWS);
    return g;
  };
  // pages of the wavefront's keys: lane l has that of tile l % NT of its keys in unit b + l / NT
  auto pages_from = [&](const Segment& g, int b) {
    const int key = (b + lane / NT) * UNIT + wave * KW + (lane % NT) * 16;
    return (c.table + (long long)g.s * c.ld_table)[min(key >> c.page_log2, c.ld_table - 1)];      // brought into its range where it is used, not to wait for it here
  };
  // A segment's queries: asked for while the one before is worked on, then turned round through LDS; a wavefront has a fourth of the channels.
  // Of 4 bits, products of bf16 have channel j beside j + 4.
  struct Queries { E x[W]; };
  struct Row { int token, head; };
  auto row_of = [&](const Segment& g, int r) {
    const int at = g.rt * ROWS + min(r, g.rows - 1), token = at / g.group;
    return Row{token, heads.head(g.kv, at - token * g.group)};
  };
  auto ask_queries = [&](const Segment& g) {
    Queries q;
    const Row r = row_of(g, n16);
    int width = dh, first = (4 * wave + quad) * W;
    asm volatile("" : "+s"(width), "+v"(first));          // what this works out is not worth registers for the rest of the kernel
    const E* from = (const E*)p.Q + (long long)r.head * dh * p.ldq + g.begin + r.token;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const int at = first + j, ch = BF && Q4 ? (at & ~7) + ((at & 7) >> 1) + 4 * (at & 1) : at;
      q.x[j] = from[(long long)(ch < width ? ch : 0) * p.ldq];
    }
    return q;
  };
  auto put_queries = [&](const Queries& q) {
    typedef E vec __attribute__((ext_vector_type(W)));
    vec v;
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = ((4 * wave + quad) * W + j & ~7) < dh ? q.x[j] : (E)0.0f;      // (heads are whole eights)
    *(vec*)&sQ[n16][(4 * wave + quad) * W] = v;
  };
  const int in_page = (1 << c.page_log2) - 1;

  // Units asked for ahead: of 4 bits one is too little to hide the way from memory (eight sequences of 33000 keys, 32 heads of 128 on 8: 84 us instead of 92, before shorter code made it 78).
  constexpr int AHEAD = BF && Q4 && W > 2 ? 2 : 1;
  const Numbers16 with_16;
  struct Tiles {
    TileT t[NT];
    __device__ __forceinline__ TileT& operator[](int i) { return t[i]; }
  };
  Tiles T[AHEAD];
  Segment g{}, next{};
  Queries queries{};
  int next_ids = 0;
  bool begun = false, first = false, loaded = false;      // loaded: the segment's first keys and values are here or on their way
  while (true) {
    if (begun && u >= u1) break;
    g = next;
    int ids = next_ids, bt = g.b0;
    if (begun) u += g.all;                 // where the next one begins
    if (u < u1) next = segment_at(u);
    // a share may begin or end among the units that a tile counts beyond its keys
    while (u < u1 && next.b1 == 0) {
      u += next.all;
      if (u < u1) next = segment_at(u);
    }
    const bool follows = u < u1;
    if (!begun) {
      if (!follows) break;
      next_ids = pages_from(next, next.b0);
      queries = ask_queries(next);
      begun = first = true;
      continue;
    }
    const int b0 = g.b0, b1 = g.b1, kv = g.kv, group = g.group, rows = g.rows;
    const Row row = row_of(g, n16);
    const int token = row.token, head = row.head;
    const int see = min(g.past + token, g.keys - 1);                                           // the row's last key
    const int see_all = min(g.past + g.rt * ROWS / group, g.keys - 1), see_any = min(g.past + (g.rt * ROWS + rows - 1) / group, g.keys - 1);
    const long long out = (long long)head * dh * p.ldc + g.begin + token;

    // the wavefront's units that some row sees
    const int keys_of_wave = see_any - wave * KW;
    const int be = keys_of_wave < 0 ? b0 : min(b1, keys_of_wave / UNIT + 1);

    // the rows of the cache that the wavefront's tiles of unit b begin at
    struct Places { long long row[NT]; };
    auto places = [&](int of, int kv_head, int b, int from) {
      Places x;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int page = clamped(__builtin_amdgcn_readlane(of, NT * (b - from) + t), 0, c.pages - 1);
        x.row[t] = (((long long)page * c.kv_heads + kv_head) << c.page_log2) + ((b * UNIT + wave * KW + t * 16) & in_page);
      }
      return x;
    };
    auto load_k = [&](const Places& at, Tiles& T) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const long long row = at.row[t];
        if constexpr (!Q4) {
          const auto g = opaque((const char*)p.K + row * (dh * (int)sizeof(E)));
          constexpr int CH = BF ? 32 : 16, LN = CH / 4;
#pragma unroll
          for (int i = 0; i < NC; ++i) {
            const int ch = CH * i + LN * quad;
            T[t].k[i] = *(Global<typename TileT::Key>)(g + (unsigned)(n16 * dh + (ch < dh ? ch : 0)) * (unsigned)sizeof(E));
          }
        } else {
          const auto g = opaque((const char*)p.K + row * (dh / 2));
          if (dh == DH) {
            typedef unsigned vec __attribute__((ext_vector_type(NC)));
            const vec x = *(Global<vec>)(g + (unsigned)(n16 * (DH / 2) + 4 * NC * quad));
#pragma unroll
            for (int i = 0; i < NC; ++i) {
              if constexpr (NC == 1) T[t].k[i] = x[0];
              else T[t].k[i] = x[i];
            }
          } else {
#pragma unroll
            for (int i = 0; i < NC; ++i) {
              const int ch = 32 * i + 8 * quad;
              T[t].k[i] = *(Global<unsigned>)(g + (unsigned)(n16 * (dh / 2) + (ch < dh ? ch : 0) / 2));
            }
          }
          const auto sc = (Global<floatx4>)(opaque(p.sK + (row >> 1)) + 32u * (unsigned)quad);
          T[t].ks[0] = sc[0];
          T[t].ks[1] = sc[1];
        }
      }
    };
    auto load_v = [&](const Places& at, Tiles& T) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const long long row = at.row[t];
        const int ch = W * n16 < dh ? W * n16 : 0;
        const auto rows_at = opaque((const char*)p.V + (Q4 ? row * (dh / 2) : row * (dh * (int)sizeof(E))));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (!Q4) {
            const auto g = rows_at + (unsigned)((4 * quad + e) * dh + ch) * (unsigned)sizeof(E);
            if constexpr (BF) {
              typedef unsigned vec __attribute__((ext_vector_type(W / 2)));
              const vec x = *(Global<vec>)g;
#pragma unroll
              for (int j = 0; j < W / 2; ++j) {
                if constexpr (W == 2) T[t].v[e][j] = x[0];
                else T[t].v[e][j] = x[j];
              }
            } else {
              constexpr int PART = W < 4 ? W : 4;
              typedef float vec __attribute__((ext_vector_type(PART)));
#pragma unroll
              for (int i = 0; i < W; i += PART) {
                const vec x = *(Global<vec>)(g + 4 * i);
#pragma unroll
                for (int j = 0; j < PART; ++j) T[t].v[e][i + j] = x[j];
              }
            }
          } else {
            const auto g = rows_at + (unsigned)((4 * quad + e) * (dh / 2) + ch / 2);
            if constexpr (W == 8) T[t].v[e] = *(Global<unsigned>)g;
            else if constexpr (W == 4) T[t].v[e] = *(Global<unsigned short>)g;
            else T[t].v[e] = *(Global<unsigned char>)g;
          }
        }
        if constexpr (Q4) {
          const auto sc = (Global<floatx4>)(opaque(p.sV + (row >> 1)) + 32u * (unsigned)quad);
          T[t].vs[0] = sc[0];
          T[t].vs[1] = sc[1];
        }
      }
    };

    auto load = [&](const Places& at, Tiles& T) {
      load_k(at, T);
      load_v(at, T);
    };
    if (!loaded) load(places(ids, kv, b0, b0), T[0]);
    if (first) {
      put_queries(queries);
      __syncthreads();
      first = false;
    }
    if (follows) {
      next_ids = pages_from(next, next.b0);
      queries = ask_queries(next);
    }
    if constexpr (AHEAD == 2) {
      if (b0 + 1 < be) {
        if (!loaded) load(places(ids, kv, b0 + 1, b0), T[1]);
      } else if (b0 < be && follows) {
        load(places(next_ids, next.kv, next.b0, next.b0), T[1]);           // (a segment of one unit: what was asked for before it was none of the next one's)
      }
    }
    // the row's query as the second operand; of 4 bits a lane has channels 8 NC apart where its heads are whole
    uintx4 qb[BF ? NC : 1];
    float qf[BF ? 1 : (Q4 ? NC * 8 : NC * 4)];
    float qsum = 0.0f;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int eight = Q4 && dh == DH ? NC * quad + i : 4 * i + quad;
      if constexpr (BF) {
        qb[i] = *(const uintx4*)&sQ[n16][8 * eight];
        if constexpr (Q4)
#pragma unroll
          for (int d = 0; d < 4; ++d) qsum += __builtin_bit_cast(float, qb[i][d] << 16) + __builtin_bit_cast(float, qb[i][d] & 0xffff0000u);
      } else {
        constexpr int PER = Q4 ? 8 : 4;
#pragma unroll
        for (int j = 0; j < PER; j += 4) {
          const floatx4 x = *(const floatx4*)&sQ[n16][PER * eight + j];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            qf[i * PER + j + e] = x[e];
            if constexpr (Q4) qsum += x[e];
          }
        }
      }
    }
    if constexpr (Q4) qsum = quads_sum(qsum);

    floatx4 O[W];
    float m, l, lowest;
    floatx4 weight;                        // of 4 bits: lowest: the sum of p lowest; weight, in each entry: of what the whole numbers were multiplied by, to take 16 off again
    bool careful = false, odd;
    while (true) {
      odd = false;
#pragma unroll
      for (int j = 0; j < W; ++j) O[j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
      m = -INFINITY;
      l = lowest = 0.0f;
      weight = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
      auto unit = [&](int b, Tiles& T) {
        const int k0 = b * UNIT + wave * KW;
        floatx4 S[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const float from = BF && Q4 ? -16.0f * qsum : 0.0f;
          S[t] = floatx4{from, from, from, from};
          if constexpr (BF && !Q4) {
#pragma unroll
            for (int i = 0; i < NC; ++i) {
              uintx4 k = T[t].k[i];
              if (32 * i + 32 > dh) {
                const unsigned keep = 32 * i + 8 * quad < dh ? ~0u : 0u;
                k &= uintx4{keep, keep, keep, keep};
              }
              S[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, qb[i]), S[t], 0, 0, 0);
            }
          } else if constexpr (BF) {
#pragma unroll
            for (int i = 0; i < NC; ++i) {
              const unsigned x = T[t].k[i];
              const uintx4 k = uintx4{with_16(x, 0), with_16(x, 1), with_16(x, 2), with_16(x, 3)};
              S[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, qb[i]), S[t], 0, 0, 0);
            }
          } else if constexpr (!Q4) {
#pragma unroll
            for (int i = 0; i < NC; ++i)
              if (16 * i < dh)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  float k = T[t].k[i][e];
                  if (16 * i + 16 > dh) k = 16 * i + 4 * quad < dh ? k : 0.0f;
                  S[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(k, qf[4 * i + e], S[t], 0, 0, 0);
                }
          } else {
#pragma unroll
            for (int i = 0; i < NC; ++i)
#pragma unroll
              for (int e = 0; e < 8; ++e)
                S[t] = __builtin_amdgcn_mfma_f32_16x16x4f32((float)(T[t].k[i] >> (4 * e) & 15u), qf[8 * i + e], S[t], 0, 0, 0);
          }
          if constexpr (Q4)
#pragma unroll
            for (int e = 0; e < 4; ++e) S[t][e] = __builtin_fmaf(S[t][e], T[t].ks[e >> 1][2 * (e & 1) + 1], qsum * T[t].ks[e >> 1][2 * (e & 1)]);
        }
        // the unit that these registers are for next, or one of the next segment's
        const bool more = b + AHEAD < be;
        Places to;
        if (more) {
          if (b + AHEAD - bt == 64 / NT) {
            bt = b + AHEAD;
            ids = pages_from(g, bt);
          }
          to = places(ids, kv, b + AHEAD, bt);
        } else if (follows) {
          to = places(next_ids, next.kv, next.b0 + (b + AHEAD - be), next.b0);
        } else {
#pragma unroll
          for (int t = 0; t < NT; ++t) to.row[t] = 0;      // what all read at their ends: were these loads left out, those before them would have to be waited for together
        }
        load_k(to, T);
        // the softmax: lane (row, quad) has the keys 4 quad .. + 4 of both tiles
        const bool whole = k0 + KW - 1 <= see_all;
        if (!whole)
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool seen = k0 + 16 * t + 4 * quad + e <= see;
              S[t][e] = seen ? S[t][e] : -INFINITY;
              if constexpr (Q4) {          // lowest and step of a key that is not seen may be anything, and would meet a probability of zero
                T[t].vs[e >> 1][2 * (e & 1)] = seen ? T[t].vs[e >> 1][2 * (e & 1)] : 0.0f;
                T[t].vs[e >> 1][2 * (e & 1) + 1] = seen ? T[t].vs[e >> 1][2 * (e & 1) + 1] : 0.0f;
              }
            }
        float mt = m;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) mt = __builtin_elementwise_maximum(mt, S[t][e]);
        mt = quads_max(mt);
        const bool grown = !((mt - m) * p.scale_log2e <= 8.0f || mt == -INFINITY);      // until then what the row holds stays as it is
        if (__builtin_amdgcn_ballot_w64(grown)) {
          const float fac = grown ? between<BF>(m, mt, p.scale_log2e) : 1.0f;
          l *= fac;
          weight *= fac;
          lowest *= fac;
#pragma unroll
          for (int j = 0; j < W; ++j) O[j] *= fac;
          m = grown ? mt : m;
        }
        const float ref = m == -INFINITY ? 0.0f : m;
        [[maybe_unused]] float ref_log2 = ref * p.scale_log2e;
        if constexpr (BF) {
          const bool far = !(fabsf(ref_log2) < FAR);
          if (__builtin_amdgcn_ballot_w64(far)) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int e = 0; e < 4; ++e) S[t][e] -= far ? ref : 0.0f;
            ref_log2 = far ? 0.0f : ref_log2;
          }
        }
        float P[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (BF) P[t][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[t][e], p.scale_log2e, -ref_log2));
            else P[t][e] = __builtin_amdgcn_exp2f((S[t][e] - ref) * p.scale_log2e);      // the difference first: it is exact, or small against what it is taken from
            if constexpr (!BF || SPLIT || Q4) l += P[t][e];
            if constexpr (Q4) {
              lowest = __builtin_fmaf(P[t][e], T[t].vs[e >> 1][2 * (e & 1)], lowest);
              P[t][e] *= T[t].vs[e >> 1][2 * (e & 1) + 1];
            }
          }
        // Values.  Where some key is not seen by every row, a value that is not finite would reach those too, by a probability of zero:
        // such values are left out of the products and added to the results of the rows that see them.
        const bool check = !Q4 && (careful || !whole);
        if constexpr (BF) {
          uintx4 hi, lo;
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const float x0 = P[d >> 1][2 * (d & 1)], x1 = P[d >> 1][2 * (d & 1) + 1];
            if constexpr (SPLIT) {
              // hi has the upper 16 bits and lo what that leaves: together within 2^-16
              const unsigned b0_ = __builtin_bit_cast(unsigned, x0), b1_ = __builtin_bit_cast(unsigned, x1);
              hi[d] = pick(b0_, b1_, HIGHS);
              const float h0 = __builtin_bit_cast(float, b0_ & 0xffff0000u), h1 = __builtin_bit_cast(float, b1_ & 0xffff0000u);
              const bf16x2 rest = bf16x2{(__bf16)(x0 - h0), (__bf16)(x1 - h1)};
              lo[d] = __builtin_bit_cast(unsigned, rest);
            } else {
              const bf16x2 one = bf16x2{(__bf16)x0, (__bf16)x1};
              hi[d] = __builtin_bit_cast(unsigned, one);
              if constexpr (!Q4) l += (float)one[0] + (float)one[1];
            }
          }
          if constexpr (Q4) {
            const uintx4 ones = uintx4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
            weight = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ones), __builtin_bit_cast(bf16x8, hi), weight, 0, 0, 0);
            if constexpr (SPLIT) weight = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ones), __builtin_bit_cast(bf16x8, lo), weight, 0, 0, 0);
          }
          if constexpr (!Q4) {
            if (check)
#pragma unroll
              for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                  for (int j = 0; j < W / 2; ++j) {
                    const unsigned x = T[t].v[e][j];
                    const bool a = (x & 0x7f80u) == 0x7f80u, z = (x & 0x7f800000u) == 0x7f800000u;
                    odd = odd || a || z;
                    T[t].v[e][j] = (a ? 0u : x & 0xffffu) | (z ? 0u : x & 0xffff0000u);
                  }
          }
#pragma unroll
          for (int j = 0; j < W; ++j) {
            uintx4 v;
#pragma unroll
            for (int d = 0; d < 4; ++d) {      // keys 2 d and 2 d + 1 of the lane's eight
              if constexpr (!Q4) {
                v[d] = pick(T[d >> 1].v[2 * (d & 1)][j >> 1], T[d >> 1].v[2 * (d & 1) + 1][j >> 1], j & 1 ? HIGHS : LOWS);
              } else {
                const unsigned a = T[d >> 1].v[2 * (d & 1)], z = T[d >> 1].v[2 * (d & 1) + 1];
                v[d] = with_16(pick(a, z, j < 4 ? LOWS : HIGHS), j & 3);
              }
            }
            O[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, hi), O[j], 0, 0, 0);
            if constexpr (SPLIT) O[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, lo), O[j], 0, 0, 0);
            if (j % 2) __builtin_amdgcn_sched_barrier(0);      // not every operand at once, for the registers
          }
        } else {
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int j = 0; j < W; ++j) {
                float v;
                if constexpr (Q4) {
                  v = (float)(T[t].v[e] >> (4 * j) & 15u);
                } else {
                  v = T[t].v[e][j];
                  if (check) {
                    const bool fin = fabsf(v) < INFINITY;
                    odd = odd || !fin;
                    v = fin ? v : 0.0f;
                  }
                }
                O[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, P[t][e], O[j], 0, 0, 0);
              }
        }
        load_v(to, T);
      };
#pragma unroll 1
      for (int b = b0; b < be; b += AHEAD) {
        unit(b, T[0]);
        if constexpr (AHEAD == 2)
          if (b + 1 < be) unit(b + 1, T[1]);
      }
      if constexpr (AHEAD == 2)
        if (b0 < be && (be - b0) % 2) {
          const Tiles x = T[0];
          T[0] = T[1];
          T[1] = x;
        }
      if constexpr (!Q4) {
        if (__builtin_amdgcn_ballot_w64(odd)) {
          // rare: the values of the blocks that were looked at once more, key by key, those that are not finite to the rows that see them
#pragma unroll 1
          for (int b = b0; b < be; ++b) {
            const int k0 = b * UNIT + wave * KW;
            if (!careful && k0 + KW - 1 <= see_all) continue;
#pragma unroll 1
            for (int key = k0; key < k0 + KW && key <= see_any; ++key) {
              int width = dh, from = 4 * W * quad;
              asm volatile("" : "+s"(width), "+v"(from));
              const int page = clamped((c.table + (long long)g.s * c.ld_table)[min(key >> c.page_log2, c.ld_table - 1)], 0, c.pages - 1);
              const E* values = (const E*)p.V + ((((long long)page * c.kv_heads + kv) << c.page_log2) + (key & in_page)) * dh;
#pragma unroll
              for (int j = 0; j < W; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const int ch = from + W * e + j;
                  const float v = (float)values[ch < width ? ch : 0];
                  O[j][e] += key <= see && !(fabsf(v) < INFINITY) ? v : 0.0f;
                  __builtin_amdgcn_sched_barrier(0);
                }
            }
          }
        }
      }
      if (Q4 || careful) break;
      // a value that is not finite and was seen by all has met a probability, or a part of one, that may be zero: the keys once more, looking at every value
      float most = 0.0f;
#pragma unroll
      for (int j = 0; j < W; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) most = __builtin_elementwise_maximum(most, fabsf(O[j][e]));
      if (!__builtin_amdgcn_ballot_w64(!(most < INFINITY))) break;
      careful = true;
      if (b0 < be) {
        bt = b0;
        ids = pages_from(g, b0);
        load(places(ids, kv, b0, b0), T[0]);
      }
    }
    loaded = follows && b0 < be;

    // ---- the four wavefronts together ----
    l = quads_sum(l);
    if constexpr (Q4) {
      lowest = quads_sum(lowest);
      if constexpr (BF) lowest -= 16.0f * weight[0];
#pragma unroll
      for (int j = 0; j < W; ++j) O[j] += lowest;
    }
    __syncthreads();                       // the segment before has been read, and this one's queries
    if (follows) put_queries(queries);
    if (quad == 0) {
      sM[wave][n16] = m;
      sL[wave][n16] = l;
      if (wave == 0) sOff[n16] = n16 < rows ? out : -1;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int j = 0; j < W; ++j) sO[wave][n16][W * (4 * quad + e) + j] = O[j][e];
    __syncthreads();
    {
      const int row = tid & 15;
      float f[4], M = sM[0][row], L = 0.0f;
#pragma unroll
      for (int w = 1; w < 4; ++w) M = __builtin_elementwise_maximum(M, sM[w][row]);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float mw = sM[w][row];
        f[w] = mw == -INFINITY ? 0.0f : between_exactly<BF>(mw, M, p.scale_log2e);      // a wavefront that saw no key has zeros
        L += f[w] * sL[w][row];
      }
      const bool whole_row = b0 == 0 && b1 == g.units;
      const long long to = sOff[row];
      const int slot = worker * 2 + (b0 == 0 ? 1 : 0);
      if (to >= 0) {
        const float inv = 1.0f / L;
        for (int ch = tid >> 4; ch < dh; ch += 16) {
          const float x = f[0] * sO[0][row][ch] + f[1] * sO[1][row][ch] + f[2] * sO[2][row][ch] + f[3] * sO[3][row][ch];
          if (whole_row) ((E*)p.C)[to + (long long)ch * p.ldc] = (E)(x * inv);
          else p.part[((long long)slot * ROWS + row) * dh + ch] = x;
        }
        if (!whole_row && tid < 16) {
          p.ml[slot * ROWS + row] = float2{M, L};
          p.off[slot * ROWS + row] = to;
        }
      }
      // the workgroups from this one to that with the tile's last unit
      if (!whole_row && b0 == 0 && tid == 0) p.parts[worker] = (int)(g.last / per) - worker + 1;
    }
  }
}

// The map of heads by workgroup, in LDS.
struct MapLds {
  unsigned short order[MAX_CACHE_HEADS];
  int first[MAX_CACHE_HEADS + 1];
};
__device__ __forceinline__ Heads heads_of(const RowsP& p, MapLds& lds, int* of) {      // of: room for MAX_CACHE_HEADS
  if (!p.kv_of_head) return Heads{nullptr, nullptr, p.group};
  const int tid = threadIdx.x;
  for (int h = tid; h < p.heads; h += 256) of[h] = clamped(p.kv_of_head[h], 0, p.c.kv_heads - 1);
  __syncthreads();
  for (int h = tid; h < p.heads; h += 256) {
    int at = 0;
    for (int o = 0; o < p.heads; ++o) at += of[o] < of[h] || (of[o] == of[h] && o < h);
    lds.order[at] = (unsigned short)h;
  }
  for (int g = tid; g <= p.c.kv_heads; g += 256) {
    int at = 0;
    for (int o = 0; o < p.heads; ++o) at += of[o] < g;
    lds.first[g] = at;
  }
  __syncthreads();
  return Heads{lds.order, lds.first, p.group};
}

template <typename E, bool Q4, int W, bool SPLIT>
__global__ __launch_bounds__(256, 2) void cache_rows_kernel(const RowsP p) {
  __shared__ __attribute__((aligned(16))) unsigned char smem[sizeof(RowsLds<W>)];
  __shared__ MapLds map;
  static_assert(sizeof(RowsLds<W>) >= 4 * MAX_CACHE_HEADS, "room for the map");
  const Heads heads = heads_of(p, map, (int*)smem);
  rows_share<E, Q4, W, SPLIT>(p, heads, smem, blockIdx.x);
}
template <bool Q4, int W, bool SPLIT>
__global__ __launch_bounds__(256, 2) void cache_wide_kernel(const RowsP p) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[Wide<W, Q4>::BYTES];
  __shared__ MapLds map;
  const Heads heads = heads_of(p, map, (int*)smem);
  wide_share<W, SPLIT, Q4>(p, heads, smem, blockIdx.x);
}

// The parts of tiles that several workgroups had, in the order of the keys.  A workgroup for a row of the tile that begins in a workgroup of the first kernel: a wavefront has a fourth of
// the parts, a lane two channels.
template <typename E>
__global__ __launch_bounds__(256) void cache_join_kernel(const RowsP p) {
  __shared__ float sO[4][128];
  __shared__ float sM[4], sL[4];
  // a tile's workgroups are on different XCDs: what one reads for itself comes an eighth as fast (105 tokens, 6 heads, on 31000 keys of 4 bits: join 34 us on one, 26 on all)
  const int worker = (int)(blockIdx.x + blockIdx.y) & (WORKERS - 1);
  if (sizeof(E) == 2 && blockIdx.x >= (unsigned)WORKERS) {
    if constexpr (sizeof(E) == 2) wide_join(p, worker, (int)blockIdx.y);
    return;
  }
  const int row = (int)blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long first = (long long)worker * 2 + 1, to = p.off[first * ROWS + row];
  const int parts = p.parts[worker];
  if (parts == 0 || to < 0) return;
  const int dh = p.c.dh, ch = 2 * lane;
  float m = -INFINITY, l = 0.0f, o[2] = {0.0f, 0.0f};
  constexpr int UN = 4;
  for (int i0 = wave; i0 < parts; i0 += 4 * UN) {
    float2 ml[UN], x[UN];
#pragma unroll
    for (int k = 0; k < UN; ++k) {
      const int i = i0 + 4 * k;
      const long long at = (i == 0 ? first : (long long)(worker + min(i, parts - 1)) * 2) * ROWS + row;
      ml[k] = p.ml[at];
      x[k] = *(const float2*)(p.part + at * dh + (ch < dh ? ch : 0));
      if (i >= parts) ml[k] = float2{-INFINITY, 0.0f};
    }
    float most = m;
#pragma unroll
    for (int k = 0; k < UN; ++k) most = __builtin_elementwise_maximum(most, ml[k].x);
    const auto factor = [&](float of) { return of == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((of - most) * p.scale_log2e); };
    const float f = factor(m);
    m = most;
    l *= f;
    o[0] *= f;
    o[1] *= f;
#pragma unroll
    for (int k = 0; k < UN; ++k) {
      const float g = factor(ml[k].x);
      if (g == 0.0f && i0 + 4 * k >= parts) continue;      // not 0 times whatever lies there
      l += g * ml[k].y;
      o[0] += g * x[k].x;
      o[1] += g * x[k].y;
    }
  }
  sO[wave][ch] = o[0];
  sO[wave][ch + 1] = o[1];
  if (lane == 0) {
    sM[wave] = m;
    sL[wave] = l;
  }
  __syncthreads();
  if ((int)threadIdx.x >= dh) return;
  float most = sM[0], sum = 0.0f, L = 0.0f;
#pragma unroll
  for (int w = 1; w < 4; ++w) most = __builtin_elementwise_maximum(most, sM[w]);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float f = sM[w] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((sM[w] - most) * p.scale_log2e);
    L += f * sL[w];
    sum += f * sO[w][threadIdx.x];
  }
  ((E*)p.C)[to + (long long)threadIdx.x * p.ldc] = (E)(sum / L);
}

struct RowsBytes { size_t part, ml, off, wide_part, wide_ml, wide_off, parts; };
static RowsBytes rows_bytes(int dh) {
  const size_t rows = (size_t)WORKERS * 2 * ROWS, wide = (size_t)WORKERS * 2 * WIDE;
  return RowsBytes{rows * dh * 4, rows * sizeof(float2), rows * 8, wide * dh * 4, wide * sizeof(float2), wide * 8, (size_t)WORKERS * 4};
}
static size_t up256(size_t b) { return (b + 255) & ~size_t(255); }

template <typename E, bool Q4, bool SPLIT>
static void launch_rows(strp_ctx* ctx, const RowsP& p, int join_rows) {
  const dim3 grid((unsigned)WORKERS), block(256);
  const auto go = [&](auto width) {
    constexpr int W = decltype(width)::value;
    if constexpr (sizeof(E) == 2)
      if (p.wide) hipLaunchKernelGGL((cache_wide_kernel<Q4, W, SPLIT>), grid, block, 0, ctx->stream, p);
    hipLaunchKernelGGL((cache_rows_kernel<E, Q4, W, SPLIT>), grid, block, 0, ctx->stream, p);
  };
  if (p.c.dh <= 32) go(std::integral_constant<int, 2>());
  else if (p.c.dh <= 64) go(std::integral_constant<int, 4>());
  else go(std::integral_constant<int, 8>());
  hipLaunchKernelGGL((cache_join_kernel<E>), dim3((unsigned)(p.wide ? 2 * WORKERS : WORKERS), (unsigned)join_rows), block, 0, ctx->stream, p);
}

}  // namespace strp

using namespace strp;

extern "C" {

size_t strp_cache_attention_workspace_bytes(int32_t d_head) {
  if (d_head <= 0 || d_head > 128) return 0;
  const RowsBytes b = rows_bytes(d_head);
  return 256 + up256(b.part) + up256(b.ml) + up256(b.off) + up256(b.wide_part) + up256(b.wide_ml) + up256(b.wide_off) + 2 * up256(b.parts);
}

strp_status strp_cache_attention(strp_ctx* ctx, const strp_cache_attention_in* in) {
  if (!ctx) return STRP_EINVAL;
  if (!in || !in->Q || !in->C) return fail(ctx, STRP_EINVAL, "cache_attention: null Q or C");
  const strp_cache& c = in->cache;
  if (const char* e = cache_error(c, in->dtype, in->heads, in->T)) return fail(ctx, STRP_EINVAL, "cache_attention: %s", e);
  if (in->T * in->heads > (1LL << 30)) return fail(ctx, STRP_EINVAL, "cache_attention: T * heads above 2^30");
  if (!in->kv_of_head && in->heads % c.kv_heads) return fail(ctx, STRP_EINVAL, "cache_attention: kv_heads does not divide heads and kv_of_head is null");
  if (!(in->scale > 0.0f) || !(in->scale <= 2.0e38f)) return fail(ctx, STRP_EINVAL, "cache_attention: scale must be positive and at most 2e38");
  if (!token_ld(in->ldq, in->T) || !token_ld(in->ldc, in->T)) return fail(ctx, STRP_EINVAL, "cache_attention: leading dimensions must be multiples of 8 and not below T");
  if (!ptr16(in->Q) || !ptr16(in->C)) return fail(ctx, STRP_EINVAL, "cache_attention: Q or C not 16-byte aligned");
  if (!ctx->ws) return fail(ctx, STRP_ENOMEM, "cache_attention: no workspace set");
  Arena arena(ctx);
  const RowsBytes b = rows_bytes(c.d_head);
  STRP_TAKE(ctx, arena, part, float, b.part / 4);
  STRP_TAKE(ctx, arena, ml, float2, b.ml / sizeof(float2));
  STRP_TAKE(ctx, arena, off, long long, b.off / 8);
  STRP_TAKE(ctx, arena, parts, int, b.parts / 4);
  STRP_TAKE(ctx, arena, wide_part, float, b.wide_part / 4);
  STRP_TAKE(ctx, arena, wide_ml, float2, b.wide_ml / sizeof(float2));
  STRP_TAKE(ctx, arena, wide_off, long long, b.wide_off / 8);
  STRP_TAKE(ctx, arena, wide_parts, int, b.parts / 4);
  OnDevice on(ctx);
  if (!on.ok()) return fail(ctx, STRP_EHIP, "cache_attention: device %d cannot be made current", ctx->device);
  RowsP p{pages_of(c, in->T), in->Q, in->C, c.K, c.V, (const floatx4*)c.K_scale, (const floatx4*)c.V_scale, in->kv_of_head, in->heads, in->heads / c.kv_heads,
          in->ldq, in->ldc, in->scale * LOG2E, 1, 4, 0, part, ml, off, parts, wide_part, wide_ml, wide_off, wide_parts};
  if (p.group == 0) p.group = 1;
  // a tile has no more rows than the heads that one key-value head can have times the tokens
  const long long rows = (in->kv_of_head ? in->heads : p.group) * in->T;
  // 128 rows at a time pay from about 2^23 pairs of a row and a key on, as far as the host knows them: what a call has beyond a token a sequence, and keys that a table has room for.  That is
  // more than there are where tables are wide (64 tokens of one sequence on 2000 keys 31 us with a table for those, 47 with one for 32768; the drafts below 114 and 118, the second launch
  // finding nothing), and fewer rows where sequences have no tokens; the kernels know better, but not before they are launched.  Below, a
  // second launch and the join of large parts cost more than reading keys again for every 16 rows (32 heads of 128 on 2000 keys each: 64 tokens of one sequence 32 us by 16, 45 by 128,
  // 5 drafts of each of 16 sequences 103 and 108, 128 tokens 46 and 49; 200 tokens 62 and 54, 33 of each of 8 sequences 141 and 79, 100 on 30000 keys 456 and 155).
  const long long beyond = rows / in->T > WIDE_FROM ? in->T : in->T - c.n_seq;
  p.wide = in->dtype == STRP_BF16 && rows > WIDE_FROM && (double)beyond * in->heads * p.c.cap >= (double)(1 << 23);
  const int join_rows = rows < ROWS ? (int)rows : ROWS;
  // the lengths are on the device: the operations and bytes of a cache that is full
  const double keys = (double)p.c.cap, T = (double)in->T, row = c.format == STRP_CACHE_Q4 ? 0.5 * c.d_head + 8.0 : bytes_of(in->dtype) * (double)c.d_head;
  ProfScope ps(ctx, "cache_attention", 4.0 * in->heads * c.d_head * T * keys, 2.0 * c.n_seq * keys * c.kv_heads * row);
  const bool q4 = c.format == STRP_CACHE_Q4;
  if (in->dtype == STRP_F32) {
    if (q4) launch_rows<float, true, false>(ctx, p, join_rows);
    else launch_rows<float, false, false>(ctx, p, join_rows);
  } else if (ctx->precision == STRP_PREC_SPLIT) {
    if (q4) launch_rows<__bf16, true, true>(ctx, p, join_rows);
    else launch_rows<__bf16, false, true>(ctx, p, join_rows);
  } else {
    if (q4) launch_rows<__bf16, true, false>(ctx, p, join_rows);
    else launch_rows<__bf16, false, false>(ctx, p, join_rows);
  }
  STRP_HIP(ctx, hipGetLastError());
  return STRP_OK;
}

}  // extern "C"
