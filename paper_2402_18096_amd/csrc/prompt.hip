// Attention of whole prompts under score rules.  Queries and keys of a prompt
// meet on the matrix cores (v_mfma_f32_32x32x16_f16, fp32 sums) one tile of 32
// keys x 32 queries at a time, in one pass over the keys with a running maximum
// and sum per query:
//   S^T = K Q^T        keys along the tile's rows, queries along its columns
//   P^T = exp2(S^T - m)
//   O^T += V^T P^T
// so a lane holds one query of a tile: its statistics are scalars, and the
// sixteen weights that it computes are, rounded to fp16, the right operand of
// the value product without leaving their registers (the order of the keys in
// that product's reduction is the one they come out in; V^T is read from LDS
// with the transposing loads in the same order).
//
// A wave holds 32 queries of one query head, two waves share a SIMD, and a block's
// waves stream the same K and V rows through LDS.  Each wave works on three subtiles
// of 32 keys at once (stage): the logits of one and the value product of another run on
// the matrix cores beside the weights of the one between.  One wave per SIMD of
// twice the queries halves the LDS reads, which are 16 % of the time there, but a wave
// issues an instruction every four to five cycles at best, and a stage has 150 of them
// beside its sixteen MFMAs of 32 cycles: with two waves they overlap.
//
// Every query sees the keys of one interval; a tile that lies inside it for all
// 32 queries takes the plain path, others are masked first.
#include <algorithm>
#include <type_traits>

#include "../../include/mikv_layer.h"
#include "prompt_device.h"

namespace mikv {

namespace {

// (lambdas with several callers over arrays in registers)
#define INLINE __attribute__((always_inline))

constexpr int kTileKeys = 64;           // keys per LDS tile
constexpr int kWaveQueries = 32;        // queries per wave of the attention
constexpr float kRaise = 1024.0f;       // raise a query's maximum when a lane's 16 weights of a tile sum past this
constexpr float kInf = __builtin_huge_valf();

struct CapPoly {
  float c0, c1, c2, c3, c4, limit;  // P's coefficients, and the |d| below which it holds
};

struct PromptArgs {
  const uint16_t *q, *k, *v;
  int64_t qs[3], ks[3], vs[3], os[3];
  uint16_t *out;
  float *lse;
  const float *slopes;
  const int32_t *begin, *end;
  int window;
  int q_heads, kv_heads, units, parts, nblk, run, T;
  float scale, cap;  // scale: of the logit in log2 units (cap: to the argument of tanh); cap in log2 units
  CapPoly poly;
};

typedef int16_t s4_t __attribute__((ext_vector_type(4)));

// The rows of a streamed tile straight to LDS, by NW waves (each wave instruction
// moves four rows), zeros past the prompt (past the descriptor's end, where rows do
// not overlap).  SWZ(row) is XORed into a row's 16-byte word index; a lane's
// offsets are the same for every tile.
template <int NW>
constexpr int tile_loads() { return kTileKeys / (4 * NW); }
struct RowOffsets {
  uint32_t at[4];
};
template <int NW, class Swz>
__device__ inline RowOffsets row_offsets(int64_t stride, Swz swz) {
  static_assert(tile_loads<NW>() <= 4, "offsets of one tile");
  RowOffsets off;
  const int lane = threadIdx.x & 63, row = 4 * (threadIdx.x >> 6) + (lane >> 4);
#pragma unroll
  for (int u = 0; u < tile_loads<NW>(); ++u) {
    const int r = row + 4 * NW * u;
    off.at[u] = (uint32_t)r * (uint32_t)(stride * 2) + 16u * (uint32_t)((lane & 15) ^ swz(r));
  }
  return off;
}
template <int NW>
__device__ inline void stage_rows(u4_t *lds, const uint16_t *rows, int64_t stride, int row0, int T,
                                  const RowOffsets &off) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), have = min(kTileKeys, T - row0);
  const __amdgpu_buffer_rsrc_t rsrc =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(rows + (int64_t)row0 * stride), (short)0,
                                        have > 0 ? (int)((have - 1) * stride * 2 + kHeadDim * 2) : 0, 0x00020000);
#pragma unroll
  for (int u = 0; u < tile_loads<NW>(); ++u)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        rsrc, (__attribute__((address_space(3))) void *)(lds + (4 * NW * u + 4 * wave) * kRowWords), 16, off.at[u], 0, 0, 0);
}
// The same through registers: fetch, and keep at the row's place.  The compiler
// waits for all loads to LDS before any LDS read that could see them, so a kernel
// whose LDS reads never pause loads its tiles this way, one tile further ahead.
template <int NW>
__device__ inline void fetch_rows(u4_t (&w)[tile_loads<NW>()], const uint16_t *rows, int64_t stride, int row0, int T) {
  const int lane = threadIdx.x & 63, row = 4 * (threadIdx.x >> 6) + (lane >> 4), have = min(kTileKeys, T - row0);
  const __amdgpu_buffer_rsrc_t rsrc =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(rows + (int64_t)row0 * stride), (short)0,
                                        have > 0 ? (int)((have - 1) * stride * 2 + kHeadDim * 2) : 0, 0x00020000);
#pragma unroll
  for (int u = 0; u < tile_loads<NW>(); ++u)
    w[u] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, (uint32_t)(row + 4 * NW * u) * (uint32_t)(stride * 2) + 16u * (uint32_t)(lane & 15), 0, 0);
}
template <int NW, class Swz>
__device__ inline void keep_rows(u4_t *lds, const u4_t (&w)[tile_loads<NW>()], Swz swz) {
  const int lane = threadIdx.x & 63, row = 4 * (threadIdx.x >> 6) + (lane >> 4);
#pragma unroll
  for (int u = 0; u < tile_loads<NW>(); ++u) {
    const int r = row + 4 * NW * u;
    lds[r * kRowWords + ((lane & 15) ^ swz(r))] = w[u];
  }
}
// K: 16 lanes read one word of 16 rows; V: 32 lanes read 32 bytes of four rows twice.
__device__ inline int swz_k(int r) { return r & 15; }
__device__ inline int swz_v(int r) { return 4 * (r & 3); }

// V^T operand of channels [32 c, 32 c + 32) and keys 16 kh .. + 15 of a 32-key
// subtile: lane l holds channel 32 c + l % 32, keys 16 kh + 4 (l / 32) + {0..3, 8..11}.
__device__ inline uint32_t v_offset() {
  const int lane = threadIdx.x & 63, i = lane & 15;
  return (uint32_t)((4 * (lane >> 5) + (i >> 2)) * 256 + 64 * (i >> 2) + 32 * ((lane >> 4) & 1) + 8 * (i & 3));
}
__device__ inline u4_t read_v(const u4_t *tile, uint32_t off, int c, int kh) {
  const char *p = reinterpret_cast<const char *>(tile) + (off ^ (64u * c)) + 256 * 16 * kh;
  typedef __attribute__((address_space(3))) s4_t *lds_s4;
  const s4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(p));
  const s4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(p + 256 * 8));
  const uint2 x = __builtin_bit_cast(uint2, a), y = __builtin_bit_cast(uint2, b);
  return u4_t{x.x, x.y, y.x, y.y};
}

// How a tile's accumulators become scores in log2 units less the query's maximum:
//   x = fma(d, P(d^2), fma(slope, row, base))
// with row the constant part of the key's index, and P the logit's scale alone
// without a cap.  CAP: where all of a tile's |d| leave tanh's argument below
// kTanhSmall, cap tanh(d arg) = d P(d^2) with P of degree four (tanh_small, its
// coefficients scaled by cap and arg once): five FMAs and a product per logit instead
// of an exponential and a reciprocal (16 cycles each) beside three of them.  A tile
// that some query does not see whole is given its final scores in the
// accumulators first (edge), and P = 1, no slope; one with a larger |d| is weighed again (settle).
struct Coef {
  float slope, base, scale, limit;
  CapPoly p;
};
__host__ __device__ constexpr float row_const(int r) { return (float)(8 * (r >> 2) + (r & 3)); }

template <bool CAP, bool BIAS>
__device__ inline float term(float d, int r, const Coef &c) {
  float a = c.base;
  if constexpr (BIAS) a = fmaf(c.slope, row_const(r), a);
  if constexpr (CAP) {
    const float u = d * d;
    return fmaf(d, fmaf(u, fmaf(u, fmaf(u, fmaf(u, c.p.c4, c.p.c3), c.p.c2), c.p.c1), c.p.c0), a);
  }
  return fmaf(d, c.scale, a);
}
// The score of a key that a query does not see.  With a cap the accumulators are
// squared: a finite number whose square is finite, below every other score
// (those end at kLowest) as -inf is.
constexpr float kLowest = -1e18f;
template <bool CAP>
constexpr float hidden_score() { return CAP ? -1.5e19f : -__builtin_huge_valf(); }

__device__ inline uint32_t pack2(float a, float b) {
  typedef _Float16 h2 __attribute__((ext_vector_type(2)));
  const h2 v = {(_Float16)a, (_Float16)b};
  return __builtin_bit_cast(uint32_t, v);
}

// One half step: the logits `next` = key x query (eight MFMAs, q), the value product
// out += vt x w (eight, v) and, between them, the weights `p` of the tile `cur`, whose
// sum is returned (CAP: infinite where a |d| is past the polynomial's limit).
//   position  0  1  2  3  4  5  6  7  8  9 10 11 12 13 14 15
//   MFMA      q0 q1 q2 v0 q3 v1 q4 v2 q5 v3 q6 v4 q7 v5 v6 v7
//   logits    0,1 2,3 4 5 6 7 8 9 10 11 12 13 14 15  -  -
// The logits end three MFMAs before the half step does, so that the next one's
// first weights need not wait for them, and the weights two before it, so that their
// sum is there when it ends.  ahead(k) issues LDS operations at position k.
template <bool CAP, bool BIAS, class Ahead>
__device__ inline float stage(f16_t &next, const u4_t (&key)[8], const u4_t (&query)[8], f16_t (&out)[4],
                              u4_t (&vt)[4][2], const u4_t (&w)[2], const f16_t &cur, const Coef &c, u4_t (&p)[2],
                              Ahead ahead) {
  f16_t d = splat(0.0f);
  float ts[2] = {0.0f, 0.0f}, big = 0.0f, x[2], e[2];
  x[0] = term<CAP, BIAS>(cur[0], 0, c);
  x[1] = term<CAP, BIAS>(cur[1], 1, c);
  int q = 0, v = 0, r = 0;  // constants once unrolled
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    if (k < 3 || (k < 13 && k % 2 == 0)) {
      d = __builtin_amdgcn_mfma_f32_32x32x16_f16(as_h8(key[q]), as_h8(query[q]), d, 0, 0, 0);
      ++q;
    } else {
      out[v & 3] = __builtin_amdgcn_mfma_f32_32x32x16_f16(as_h8(vt[v & 3][v >> 2]), as_h8(w[v >> 2]), out[v & 3], 0, 0, 0);
      ++v;
    }
    ahead(k);
    const int n = k < 2 ? 2 : k < 14 ? 1 : 0;
#pragma unroll
    for (int h = 0; h < n; ++h, ++r) {
      float pr = __builtin_amdgcn_exp2f(x[r & 1]);
      if constexpr (CAP) big = fmaxf(big, fabsf(cur[r]));
      if (r < 14) x[r & 1] = term<CAP, BIAS>(cur[r + 2], r + 2, c);
      ts[r & 1] += pr;
      // (here: the compiler would move all this behind the MFMAs)
      if (r & 1) {
        uint32_t w2 = pack2(e[0], pr);
        asm volatile("" : "+v"(w2), "+v"(ts[0]), "+v"(ts[1]), "+v"(big));
        p[r >> 3][(r >> 1) & 3] = w2;
      } else {
        asm volatile("" : "+v"(pr));
        e[0] = pr;
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  next = d;
  return CAP && !(big < c.limit) ? kInf : ts[0] + ts[1];
}

// The value of the lane 32 away (no LDS operation, which would be in the way of the loop's own).
__device__ inline float other_half(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  return __builtin_bit_cast(float, (threadIdx.x & 32) ? r[0] : r[1]);
}

// Smallest of all lanes, as a scalar (DPP inside the rows of 16, as wave_max).
__device__ inline int wave_min_int(int v) {
  v = min(v, __builtin_amdgcn_mov_dpp(v, 0xB1, 0xF, 0xF, true));
  v = min(v, __builtin_amdgcn_mov_dpp(v, 0x4E, 0xF, 0xF, true));
  v = min(v, __builtin_amdgcn_mov_dpp(v, 0x141, 0xF, 0xF, true));
  v = min(v, __builtin_amdgcn_mov_dpp(v, 0x140, 0xF, 0xF, true));
  const int a = min(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16));
  return min(a, min(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
}
__device__ inline int wave_max_int(int v) { return -wave_min_int(-v); }

// A query's interval, clamped to the prompt; empty: (0, 0).
__device__ inline void query_span(const int32_t *begin, const int32_t *end, int window, int64_t at, int i, int T, int &lo,
                                  int &hi) {
  lo = begin ? max(begin[at], 0) : 0;
  hi = end ? min(end[at], T) : i + 1;
  if (window > 0) lo = max(lo, i + 1 - min(window, i + 1));
  if (lo >= hi) lo = hi = 0;
}

// block_unit with a unit's blocks dealt out to `parts` XCDs (unit_parts).
__device__ inline bool block_of_unit(int units, int per_unit, int parts, int run, int &unit, int &idx) {
  if (!block_unit(units * parts, (per_unit + parts - 1) / parts, run, unit, idx)) return false;
  idx = idx * parts + unit % parts;
  unit /= parts;
  return idx < per_unit;
}

// A block of NW waves: min(G, NW) query heads of one KV head's group times the
// 32-query tiles that fill it, so that its waves need the same keys as nearly as
// they can.
template <bool CAP, bool BIAS, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2)))
void prompt_attention_kernel(PromptArgs A) {
  constexpr int TR = kTileKeys, kTile = TR * kRowWords;
  __shared__ u4_t s_lds[5 * kTile];  // three tiles of K, two of V
  auto k_tile = [&](int t) INLINE { return s_lds + (t % 3) * kTile; };
  auto v_tile = [&](int t) INLINE { return s_lds + (3 + (t & 1)) * kTile; };
  int(*s_span)[2] = reinterpret_cast<int(*)[2]>(s_lds + 2 * kTile);  // free until the third tile
  const int lane = threadIdx.x & 63, n = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = A.q_heads / A.kv_heads, T = A.T;
  const int hw = min(G, NW), rw = NW / hw, groups = G / hw;  // heads and query tiles of a block, head groups
  int hk, idx;
  if (!block_of_unit(A.units, A.nblk * groups, A.parts, A.run, hk, idx)) return;
  const int b = hk / A.kv_heads, kvh = hk % A.kv_heads, head = kvh * G + (idx % groups) * hw + wave % hw;
  const int i_wave = kWaveQueries * ((A.nblk - 1 - idx / groups) * rw + wave / hw);
  const uint16_t *kb = A.k + b * A.ks[0] + kvh * A.ks[1], *vb = A.v + b * A.vs[0] + kvh * A.vs[1];
  const uint16_t *qb = A.q + b * A.qs[0] + head * A.qs[1];

  // The queries, and their intervals (queries past the prompt repeat the last one).
  const int i_own = min(i_wave + n, T - 1), i_lo = min(i_wave, T - 1), i_hi = min(i_wave + 31, T - 1);
  u4_t bq[8];
  {
    const uint16_t *r = qb + (int64_t)i_own * A.qs[2] + 8 * half;
#pragma unroll
    for (int c = 0; c < 8; ++c) bq[c] = *reinterpret_cast<const u4_t *>(r + 16 * c);
  }
  int lo, hi;
  query_span(A.begin, A.end, A.window, (int64_t)b * T + i_own, i_own, T, lo, hi);
  const int full_lo = wave_max_int(lo), full_hi = wave_min_int(hi);
  const int own_lo = wave_min_int(hi ? lo : T), own_hi = wave_max_int(hi);
  if (lane == 0) {
    s_span[wave][0] = own_lo;
    s_span[wave][1] = own_hi;
  }
  __syncthreads();
  int any_lo = own_lo, any_hi = own_hi;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    any_lo = min(any_lo, s_span[w][0]);
    any_hi = max(any_hi, s_span[w][1]);
  }
  any_lo = __builtin_amdgcn_readfirstlane(any_lo);
  any_hi = __builtin_amdgcn_readfirstlane(any_hi);
  const int t_first = any_lo / TR, n_tiles = max(0, (any_hi + TR - 1) / TR - t_first);

  const float slope = BIAS ? A.slopes[head] * kLog2e : 0.0f;
  float m = -kInf, l = 0.0f;
  f16_t o[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) o[c] = splat(0.0f);

  if (n_tiles > 0) {
    // whether every query sees keys j0 .. j0 + 31, on one side of it where the bias needs that
    auto full = [&](int j0) INLINE {
      bool f = j0 >= full_lo && j0 + 32 <= full_hi;
      if constexpr (BIAS) f = f && (j0 + 31 <= i_lo || j0 > i_hi);
      return f;
    };
    auto coef = [&](bool is_full, int j0) INLINE {
      Coef c;
      c.slope = 0.0f;
      c.base = -m;
      if constexpr (CAP) {
        c.p.c0 = is_full ? A.poly.c0 : 1.0f;
        c.p.c1 = is_full ? A.poly.c1 : 0.0f;
        c.p.c2 = is_full ? A.poly.c2 : 0.0f;
        c.p.c3 = is_full ? A.poly.c3 : 0.0f;
        c.p.c4 = is_full ? A.poly.c4 : 0.0f;
        c.limit = is_full ? A.poly.limit : kInf;
      } else {
        c.scale = is_full || !BIAS ? A.scale : 1.0f;
      }
      if constexpr (BIAS) {
        c.slope = !is_full ? 0.0f : j0 > i_hi ? -slope : slope;
        c.base = fmaf(c.slope, (float)(j0 + 4 * half - i_own), c.base);
      }
      return c;
    };
    // final scores of a subtile of which not every query sees every key
    auto edge = [&](f16_t &d, int j0) INLINE {
      if (j0 >= own_hi || j0 + 32 <= own_lo) {
        d = splat(hidden_score<CAP>());
        return;
      }
      constexpr bool kEdgeScaled = !CAP && BIAS;  // (without either, term scales -inf, too)
      const int jb = j0 + 4 * half;
      if constexpr (CAP) {
        float big = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) big = fmaxf(big, fabsf(d[r]));
        Coef c;
        c.base = 0.0f;
        c.p = A.poly;
        if (__ballot(!(big < c.p.limit)) == 0) {
#pragma unroll
          for (int r = 0; r < 16; ++r) d[r] = term<true, false>(d[r], r, c);
        } else {
#pragma unroll
          for (int r = 0; r < 16; ++r) d[r] = tanh_fine(d[r] * A.scale) * A.cap;
        }
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int c = (int)row_const(r);
        float s = kEdgeScaled ? d[r] * A.scale : d[r];
        if constexpr (BIAS) s = fmaf(-slope, (float)abs(i_own - jb - c), s);
        if constexpr (CAP) s = s < kLowest ? kLowest : s;
        d[r] = (uint32_t)(jb - lo + c) < (uint32_t)(hi - lo) ? s : hidden_score<CAP>();
      }
    };
    // Whether every lane's weights of a subtile are in range.
    auto fine = [&](float ts) INLINE { return __ballot(!(ts <= kRaise)) == 0; };
    // Where a subtile's weights sum past kRaise (or are NaN: the maximum starts at
    // -inf; or not valid, see stage) in any lane: raise the maxima, rescale, and
    // weigh the subtile again.  The two lanes of a query keep one maximum.
    auto raise = [&](const f16_t &d, bool is_full, int j0, float &ts, u4_t (&p)[2]) INLINE {
      Coef c = coef(is_full, j0);
      c.base = BIAS ? c.slope * (float)(j0 + 4 * half - i_own) : 0.0f;
      float s[16], mx = -kInf;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if constexpr (CAP) {
          s[r] = is_full ? fmaf(tanh_fine(d[r] * A.scale), A.cap, BIAS ? fmaf(c.slope, row_const(r), c.base) : 0.0f)
                         : d[r] < 5.0f * kLowest ? -kInf : d[r];
        } else {
          s[r] = term<CAP, BIAS>(d[r], r, c);
        }
        mx = fmaxf(mx, s[r]);
      }
      mx = fmaxf(m, fmaxf(mx, other_half(mx)));
      const float ref = mx == -kInf ? 0.0f : mx;
      const float f = m == -kInf ? 0.0f : __builtin_amdgcn_exp2f(m - ref);
      m = mx;
      l *= f;
#pragma unroll
      for (int c4 = 0; c4 < 4; ++c4)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[c4][r] *= f;
      ts = 0.0f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = __builtin_amdgcn_exp2f(s[r] - ref);
        ts += s[r];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i >> 2][i & 3] = pack2(s[2 * i], s[2 * i + 1]);
      return f;
    };

    // The tiles pass through registers, K and V in turn: tile t + 1's keys are kept in
    // LDS during the first subtile of tile t, its value rows during the second, each
    // fetched one subtile before.  (Past the last tile rows are loaded, or zeros,
    // and never used.)
    // The tiles go backwards: under a bias the first scores are then the largest (of the
    // keys no later than the query), and the maximum is not raised at every tile (1 x 4 x 2048
    // 78 -> 52 us); packed documents gain, too (16 x 32/8 x 2011 330 -> 308, under a cap 454 ->
    // 402, 8 x 32 x 4096 1004 -> 810), other prompts are even, but under a cap alone forwards is
    // a percent faster (8 x 32 x 4096 1612 -> 1593).
    const bool back = BIAS || !CAP || A.begin || A.end;
    auto tile = [&](int t) INLINE { return back ? max(t_first + n_tiles - 1 - t, 0) : t_first + t; };
    u4_t rows[tile_loads<NW>()];
    auto fetch_keys = [&](int t) INLINE { fetch_rows<NW>(rows, kb, A.ks[2], tile(t) * TR, T); };
    auto fetch_values = [&](int t) INLINE { fetch_rows<NW>(rows, vb, A.vs[2], tile(t) * TR, T); };
    auto feed_keys = [&](int t) INLINE {
      keep_rows<NW>(k_tile(t), rows, swz_k);
      fetch_values(t);
    };
    auto feed_values = [&](int t) INLINE {
      keep_rows<NW>(v_tile(t), rows, swz_v);
      fetch_keys(t + 1);
    };
    {
      u4_t values[tile_loads<NW>()];
      fetch_keys(0);
      fetch_rows<NW>(values, vb, A.vs[2], tile(0) * TR, T);
      keep_rows<NW>(k_tile(0), rows, swz_k);
      fetch_keys(1);
      keep_rows<NW>(v_tile(0), values, swz_v);
    }
    __syncthreads();
    // A tile that this wave does not see.  At the barrier the next tile's keys and
    // this one's value rows are complete, and every wave is done with the keys of the tile
    // before and with its value rows.
    auto idle = [&](int t) INLINE {
      feed_keys(t + 1);
      __syncthreads();
      feed_values(t + 1);
    };

    // The tiles that any query of this wave sees; for the others it only keeps step
    // with the block.
    int own_first = own_hi > own_lo ? own_lo / TR - t_first : 0;
    int own_end = own_hi > own_lo ? (own_hi + TR - 1) / TR - t_first : 0;
    if (back) {
      const int first = own_first;
      own_first = n_tiles - own_end;
      own_end = n_tiles - first;
    }
    for (int t = 0; t < own_first; ++t) idle(t);

    const uint32_t off = tile_offset(), voff = v_offset();
    // Before the first subtile: weights and value operands of zero, and a subtile
    // that sees nothing (edge form).
    u4_t kf[8], vf[4][2], p0[2], p1[2];
#pragma unroll
    for (int i = 0; i < 8; ++i) vf[i & 3][i >> 2] = u4_t{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 2; ++i) p0[i] = p1[i] = u4_t{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) kf[i] = read_word(k_tile(own_first), off, 0, i);
    // A value of a row that some query does not see must not reach that query as
    // 0 x NaN: in an edge subtile infinities and NaN are taken out of the value
    // operand (clean says whether any were there), and the queries that do see
    // one become NaN in its channel (poison).
    auto odd_halves = [](uint32_t w) INLINE { return (((w & 0x7fff7fffu) + 0x04000400u) & 0x80008000u) >> 15; };  // 1 per infinite or NaN half
    auto clean = [&]() INLINE {
      // (a sum of fp16 values in fp32 is finite where they all are)
      typedef _Float16 h2 __attribute__((ext_vector_type(2)));
      float any[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t w = vf[i & 3][i >> 2][e];
          any[e] = __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, w), h2{(_Float16)1.0f, (_Float16)1.0f}, any[e], false);
        }
      if (!__ballot(!(fabsf((any[0] + any[1]) + (any[2] + any[3])) < kInf))) return false;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) vf[i & 3][i >> 2][e] &= ~(odd_halves(vf[i & 3][i >> 2][e]) * 0xffffu);
      return true;
    };
    auto poison = [&](const u4_t *v, const u4_t (&p)[2]) INLINE {
      auto ones = [](uint32_t w) INLINE { return ((w & 0xffffu) ? 0x3c00u : 0u) | ((w >> 16) ? 0x3c000000u : 0u); };
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        f16_t hits = splat(0.0f);
#pragma unroll
        for (int kh = 0; kh < 2; ++kh) {
          u4_t a = read_v(v, voff, c, kh), w = p[kh];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            a[e] = odd_halves(a[e]) * 0x3c00u;
            w[e] = ones(w[e]);
          }
          hits = __builtin_amdgcn_mfma_f32_32x32x16_f16(as_h8(a), as_h8(w), hits, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) o[c][r] += hits[r] > 0.0f ? __builtin_nanf("") : 0.0f;
      }
    };
    f16_t d0 = splat(hidden_score<CAP>()), d1;
    bool was_full = false;  // of the subtile before
    // Its first key and value rows.  Before the first subtile: rows that are complete
    // (those of the first tile come after the barrier), with weights of zero; infinities
    // and NaN are taken out of them unless every query sees them anyway.
    const int t_zero = max(own_first - 1, 0);
    int j_was = tile(t_zero) * TR;
    const u4_t *v_was = v_tile(t_zero);
    // One subtile: logits of it into `d`, weights of the one before, whose logits `was`
    // holds, into `p`, and value product of the one before that, whose weights `pv` holds.
    auto subtile = [&](auto which, int t, f16_t &d, f16_t &was, u4_t (&p)[2], u4_t (&pv)[2]) INLINE {
      constexpr int S = decltype(which)::value;  // of the tile's two
      const int j0 = tile(t) * TR + 32 * S;
      if constexpr (S == 1) __syncthreads();
      const u4_t *kt = k_tile(t), *kn = k_tile(t + S);
      auto ahead = [&](int k) INLINE {
        // this subtile's second half of the keys, the value rows of the subtile before
        // and the next one's first half of the keys, in time for their MFMAs and as the
        // operands they take the place of are done with
        if (k < 4) kf[4 + k] = read_word(kt, off, 32 * S, 4 + k);
        if (k >= 4 && k <= 10 && k % 2 == 0) vf[(k - 4) / 2][0] = read_v(v_was, voff, (k - 4) / 2, 0);
        if (k == 2) {
          if constexpr (S == 0)
            feed_keys(t + 1);
          else
            feed_values(t + 1);
        }
        if (k >= 11 && k <= 14) kf[k - 11] = read_word(kn, off, 32 * (1 - S), k - 11);
      };
      float ts = stage<CAP, BIAS>(d, kf, bq, o, vf, pv, was, coef(was_full, j_was), p, ahead);
#pragma unroll
      for (int c = 0; c < 4; ++c) vf[c][1] = read_v(v_was, voff, c, 1);
      const bool is_full = full(j0), ok = fine(ts);
      // (one branch, rarely taken, for all that is not plain)
      if (__builtin_expect(!ok || !is_full || !was_full, false)) {
        if (S == 0 && t == own_first) {  // nothing came before: m - m is not a number
          ts = 0.0f;
          p[0] = p[1] = u4_t{0, 0, 0, 0};
        } else if (!ok) {
          raise(was, was_full, j_was, ts, p);
        }
        if (!is_full) edge(d, j0);
        if (!(j_was >= full_lo && j_was + 32 <= full_hi) && clean()) poison(v_was, p);
      }
      l += ts;
      was_full = is_full;
      j_was = j0;
      v_was = v_tile(t) + 32 * S * kRowWords;
    };
    for (int t = own_first; t < own_end; ++t) {
      subtile(std::integral_constant<int, 0>{}, t, d1, d0, p0, p1);
      subtile(std::integral_constant<int, 1>{}, t, d0, d1, p1, p0);
    }
    // the weights of the last subtile, and both last value products
    auto product = [&](const u4_t (&p)[2]) INLINE {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_f16(as_h8(vf[i & 3][i >> 2]), as_h8(p[i >> 2]), o[i & 3], 0, 0, 0);
    };
    product(p1);
    {
      const Coef c = coef(was_full, j_was);
      float ts = 0.0f, big = 0.0f, x[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[r] = __builtin_amdgcn_exp2f(term<CAP, BIAS>(d0[r], r, c));
        ts += x[r];
        big = fmaxf(big, fabsf(d0[r]));
      }
      if (CAP && !(big < c.limit)) ts = kInf;
#pragma unroll
      for (int i = 0; i < 8; ++i) p0[i >> 2][i & 3] = pack2(x[2 * i], x[2 * i + 1]);
      if (!fine(ts)) raise(d0, was_full, j_was, ts, p0);
      l += ts;
    }
    if (own_first < own_end) {
#pragma unroll
      for (int i = 0; i < 8; ++i) vf[i & 3][i >> 2] = read_v(v_was, voff, i & 3, i >> 2);
      if (!(j_was >= full_lo && j_was + 32 <= full_hi) && clean()) poison(v_was, p0);
      product(p0);
    }
    for (int t = own_end; t < n_tiles; ++t) idle(t);
  }

  // out = O / l, through LDS so that whole rows are stored
  __syncthreads();
  u4_t *own_rows = s_lds + wave * (kWaveQueries * kRowWords);  // 8 KiB each
  const float sum = l + other_half(l);
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  if (A.lse && half == 0 && i_wave + n < T)
    A.lse[((int64_t)b * A.q_heads + head) * T + i_wave + n] =
        sum == 0.0f ? -kInf : (m + __builtin_amdgcn_logf(sum)) * kLn2;
  uint2 *row = reinterpret_cast<uint2 *>(own_rows) + n * (2 * kRowWords);
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const int w = 4 * c + a;  // 16-byte word: channels 32 c + 8 a ..
      row[2 * (w ^ (n & 15)) + half] = make_uint2(pack2(o[c][4 * a] * inv, o[c][4 * a + 1] * inv),
                                                 pack2(o[c][4 * a + 2] * inv, o[c][4 * a + 3] * inv));
    }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
  uint16_t *ob = A.out + b * A.os[0] + head * A.os[1];
#pragma unroll
  for (int u = 0; u < kWaveQueries / 4; ++u) {
    const int r = 4 * u + (lane >> 4), i = i_wave + r;
    const u4_t w = own_rows[r * kRowWords + ((lane & 15) ^ (r & 15))];
    if (i < T) *reinterpret_cast<u4_t *>(ob + (int64_t)i * A.os[2] + 8 * (lane & 15)) = w;
  }
}

// H2O importance under the rules: a wave holds 64 keys of one KV head and streams
// the queries of one query head past them (queries along the tile's columns, so a
// lane holds one query per tile, whose log-sum-exp and interval are scalars), as
// prefill_colsum_kernel does for the causal case.  WS waves of the block take the
// same keys and share out the 32-query subtiles.  The heads of a group have blocks
// of their own and are added up afterwards in head order: with documents the
// longest block, not the work, was the launch (8 x 32/8 x 4096, documents of up to 2500
// tokens, a cap: 717 -> 541 us).  Bound: the VALU beside the MFMAs (16 exponentials and,
// under a cap, 112 FMAs per 32 x 32 logits and lane group) at two waves per SIMD; 0.78
// PFLOP/s for 8 x 32/8 x 4096 without rules, 385 us for the documents above.
struct SumArgs {
  const uint16_t *q, *k;
  int64_t qs[3], ks[3];
  const float *lse, *slopes;
  const int32_t *begin, *end;
  const int4 *spans;  // of every 32 queries, or NULL (causal)
  float *sums;  // [batch, q_heads, T]
  int window;
  int q_heads, kv_heads, units, parts, nblk, run, T;
  float scale, cap;
  CapPoly poly;
};

// Interval extremes of 32 queries: smallest begin and largest end over those that
// see something, largest begin and smallest end over all (the latter 0 if one
// sees nothing).
__global__ __launch_bounds__(64) void query_spans_kernel(const int32_t *begin, const int32_t *end, int window, int T, int nsub,
                                                       int4 *spans) {
  const int b = blockIdx.y, i = blockIdx.x * 64 + threadIdx.x;
  int lo = 0, hi = 0;
  if (i < T) query_span(begin, end, window, (int64_t)b * T + i, i, T, lo, hi);
  int a = hi ? lo : T, z = hi, x = lo, y = hi;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a = min(a, __shfl_xor(a, o, 64));
    z = max(z, __shfl_xor(z, o, 64));
    x = max(x, __shfl_xor(x, o, 64));
    y = min(y, __shfl_xor(y, o, 64));
  }
  if ((threadIdx.x & 31) == 0 && i / 32 < nsub) spans[(int64_t)b * nsub + i / 32] = make_int4(a, z, x, y);
}

__device__ inline int4 causal_span(int i0, int T) {
  return i0 >= T ? make_int4(T, 0, 0, 0) : make_int4(0, min(i0 + 32, T), 0, i0 + 31 < T ? i0 + 1 : 0);
}

// Sums of 32 values over each half of the wave: lane n of a half gets value n's.  The
// lanes 16, 8, 4, 2 and 1 away exchange the halves of the values that the other one keeps:
// 31 exchanges (a butterfly per value takes 160).
template <int SPAN = 8>
__device__ inline float own_sum16(float (&v)[32]) {
  if constexpr (SPAN == 0) {
    return v[0];
  } else {
    const bool up = lanes_with<SPAN>();
#pragma unroll
    for (int k = 0; k < SPAN; ++k)
      v[k] = (up ? v[k + SPAN] : v[k]) +
             dpp_mov<SPAN == 8 ? 0x140 : SPAN == 4 ? 0x141 : SPAN == 2 ? 0x4E : 0xB1>(up ? v[k] : v[k + SPAN]);
    return own_sum16<SPAN / 2>(v);
  }
}
__device__ inline float own_sum32(float (&v)[32]) {
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v[k]), __builtin_bit_cast(uint32_t, v[k + 16]), false, false);
    const uint32_t x = r[0], y = r[1];
    v[k] = __builtin_bit_cast(float, x) + __builtin_bit_cast(float, y);
  }
  return own_sum16(v);
}

template <int WS>
constexpr int sum_rows() { return WS == 4 ? 128 : 64; }

template <int WS, bool CAP, bool BIAS>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2)))
void prompt_colsum_kernel(SumArgs A) {
  constexpr int TR = sum_rows<WS>(), SUBS = TR / 32 / WS, kKeys = kWaveRows * 4 / WS;
  __shared__ u4_t s_rows[2][TR * kRowWords];
  __shared__ float s_lse[2][TR];
  __shared__ int2 s_span[2][TR];
  __shared__ int4 s_sub[2][TR / 32];
  __shared__ float s_sum[4][kWaveRows];
  __shared__ int s_range[4][2];
  const int lane = threadIdx.x & 63, n = lane & 31, half = lane >> 5, tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wc = wave / WS, ws = wave % WS;
  const int G = A.q_heads / A.kv_heads, T = A.T, nsub = (T + 31) / 32;
  int hk, idx;
  if (!block_of_unit(A.units, A.nblk * G, A.parts, A.run, hk, idx)) return;
  const int b = hk / A.kv_heads, kvh = hk % A.kv_heads, head = kvh * G + idx % G;
  const int j_base = idx / G * kKeys, j_wave = j_base + kWaveRows * wc;
  const int64_t row = ((int64_t)b * A.q_heads + head) * T;  // of lse and sums
  const uint16_t *qb = A.q + b * A.qs[0] + head * A.qs[1], *kb = A.k + b * A.ks[0] + kvh * A.ks[1];
  auto sub_span = [&](int sub) {
    if (sub >= nsub) return make_int4(T, 0, 0, 0);
    return A.spans ? A.spans[(int64_t)b * nsub + sub] : causal_span(32 * sub, T);
  };
  // the query tiles between the first and the last that see any of the block's keys
  int first = nsub, last = -1;
  for (int s = tid; s < nsub; s += kThreads) {
    const int4 v = sub_span(s);
    if (v.x < j_base + kKeys && v.y > j_base) {
      first = min(first, s);
      last = s;
    }
  }
  first = wave_min_int(first);
  last = wave_max_int(last);
  if (lane == 0) {
    s_range[wave][0] = first;
    s_range[wave][1] = last;
  }
  u4_t ak[2][8];
#pragma unroll
  for (int cb = 0; cb < 2; ++cb) {
    const uint16_t *r = kb + (int64_t)min(j_wave + 32 * cb + n, T - 1) * A.ks[2] + 8 * half;
#pragma unroll
    for (int c = 0; c < 8; ++c) ak[cb][c] = *reinterpret_cast<const u4_t *>(r + 16 * c);
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    first = min(first, s_range[w][0]);
    last = max(last, s_range[w][1]);
  }
  first = __builtin_amdgcn_readfirstlane(first);
  last = __builtin_amdgcn_readfirstlane(last);
  const int t_first = 32 * first / TR, t_end = last < first ? t_first : 32 * last / TR + 1;

  const RowOffsets q_off = row_offsets<4>(A.qs[2], swz_k);
  f16_t cs[2] = {splat(0.0f), splat(0.0f)};
  float r_lse = 0.0f;
  int2 r_span = make_int2(0, 0);
  int4 r_sub = make_int4(0, 0, 0, 0);
  auto load = [&](int buf, int t) {
#pragma unroll
    for (int u = 0; u < TR / 64; ++u)
      stage_rows<4>(s_rows[buf] + 64 * u * kRowWords, qb, A.qs[2], t * TR + 64 * u, T, q_off);
    if (tid < TR) {
      const int i = t * TR + tid, ic = min(i, T - 1);
      r_lse = A.lse[row + ic] * kLog2e;
      int lo, hi;
      query_span(A.begin, A.end, A.window, (int64_t)b * T + ic, ic, T, lo, hi);
      r_span = i < T ? make_int2(lo, hi) : make_int2(0, 0);
    }
    if (tid < TR / 32) r_sub = sub_span(t * (TR / 32) + tid);
  };
  auto commit = [&](int buf) {
    if (tid < TR) {
      s_lse[buf][tid] = r_lse;
      s_span[buf][tid] = r_span;
    }
    if (tid < TR / 32) s_sub[buf][tid] = r_sub;
    wait_loads();
    __syncthreads();
  };
  const uint32_t off = tile_offset();
  if (t_first < t_end) {
    load(0, t_first);
    commit(0);
    int buf = 0;
    const float slope = BIAS ? A.slopes[head] * kLog2e : 0.0f;
    for (int t = t_first; t < t_end; ++t) {
      const u4_t *rows = s_rows[buf];
#pragma unroll
      for (int s = 0; s < SUBS; ++s) {
        const int sub = ws * SUBS + s, i0 = t * TR + 32 * sub;
        const int4 sp = s_sub[buf][sub];
        const int any_lo = __builtin_amdgcn_readfirstlane(sp.x), any_hi = __builtin_amdgcn_readfirstlane(sp.y);
        const int full_lo = __builtin_amdgcn_readfirstlane(sp.z), full_hi = __builtin_amdgcn_readfirstlane(sp.w);
        u4_t bq[8];
        read_tile(rows, off, 32 * sub, bq);
        const float lse2 = s_lse[buf][32 * sub + n];
        const int2 span = s_span[buf][32 * sub + n];
        if (s == SUBS - 1) {  // after the tile's last LDS read: the compiler holds LDS reads back for loads to LDS
          load(buf ^ 1, min(t + 1, t_end - 1));
        }
        if (any_lo >= j_wave + kWaveRows || any_hi <= j_wave) continue;  // wave-uniform
        const int i = min(i0 + n, T - 1);
#pragma unroll
        for (int cb = 0; cb < 2; ++cb) {
          const int j0 = j_wave + 32 * cb;
          if (any_lo >= j0 + 32 || any_hi <= j0) continue;
          f16_t d = logits(ak[cb], bq);
          bool full = j0 >= full_lo && j0 + 32 <= full_hi, in_poly = true;
          if constexpr (BIAS) full = full && (j0 + 31 <= i0 || j0 > i0 + 31);
          if constexpr (CAP) {
            float big = 0.0f;
#pragma unroll
            for (int r = 0; r < 16; ++r) big = fmaxf(big, fabsf(d[r]));
            in_poly = !__ballot(!(big < A.poly.limit));
          }
          if (full && in_poly) {
            Coef c = {0.0f, -lse2, A.scale, 0.0f, A.poly};
            if constexpr (BIAS) {
              c.slope = j0 > i0 ? -slope : slope;
              c.base = fmaf(c.slope, (float)(j0 + 4 * half - i), c.base);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) cs[cb][r] += __builtin_amdgcn_exp2f(term<CAP, BIAS>(d[r], r, c));
          } else {
            if (in_poly) {
              const Coef c = {0.0f, 0.0f, A.scale, 0.0f, A.poly};
#pragma unroll
              for (int r = 0; r < 16; ++r) d[r] = term<CAP, false>(d[r], r, c);
            } else {
#pragma unroll
              for (int r = 0; r < 16; ++r) d[r] = tanh_fine(d[r] * A.scale) * A.cap;
            }
            const int jb = j0 + 4 * half;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int j = jb + (int)row_const(r);
              float x = d[r];
              if constexpr (BIAS) x = fmaf(-slope, (float)abs(i - j), x);
              const float p = __builtin_amdgcn_exp2f(x - lse2);
              cs[cb][r] += (uint32_t)(j - span.x) < (uint32_t)(span.y - span.x) ? p : 0.0f;
            }
          }
        }
      }
      buf ^= 1;
      commit(buf);
    }
  }
  // over the tile's 32 query columns, then over the WS waves: lane n of a half has the
  // half's rows tile_row(n % 16) of the first (n < 16) or second 32 keys
  float v32[32];
#pragma unroll
  for (int r = 0; r < 32; ++r) v32[r] = cs[r >> 4][r & 15];
  s_sum[wave][32 * (n >> 4) + tile_row(n & 15)] = own_sum32(v32);
  __syncthreads();
  if (ws != 0) return;
  float v = s_sum[wave][lane];
#pragma unroll
  for (int o = 1; o < WS; ++o) v += s_sum[wave + o][lane];
  const int kj = j_wave + lane;
  if (kj < T) A.sums[row + kj] = v;
}

__global__ __launch_bounds__(256) void sum_heads_kernel(const float *sums, int units, int G, int T, float *scores) {
  const int j = blockIdx.x * 256 + threadIdx.x;
  const int64_t hk = (int64_t)blockIdx.z * 65535 + blockIdx.y;
  if (j >= T || hk >= units) return;
  const float *p = sums + hk * G * T + j;
  float v = p[0];
  for (int g = 1; g < G; ++g) v += p[(int64_t)g * T];
  scores[hk * T + j] = v;
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------

// The rows of one tensor: 16-byte aligned, strides multiples of 8, and a tile's
// byte offsets (64 rows) within 31 bits.
int check_rows(const char *who, const char *name, const void *p, const int64_t s[3]) {
  if (!p) return set_error(MIKV_ERR_INVALID_ARG, "%s: %s is NULL", who, name);
  if ((uintptr_t)p % 16 || s[0] % 8 || s[1] % 8 || s[2] % 8)
    return set_error(MIKV_ERR_INVALID_ARG, "%s: %s: rows must be 16-byte aligned, strides multiples of 8", who, name);
  if (s[0] < 0 || s[1] < 0 || s[2] < 0) return set_error(MIKV_ERR_INVALID_ARG, "%s: %s: negative stride", who, name);
  if (s[2] > (int64_t)1 << 22) return set_error(MIKV_ERR_UNSUPPORTED, "%s: %s: token stride over 2^22", who, name);
  return MIKV_OK;
}

int check_prompt(const char *who, const mikv_prompt *p, const mikv_score_rules *r) {
  if (!p) return set_error(MIKV_ERR_INVALID_ARG, "%s: prompt is NULL", who);
  if (p->batch < 1 || p->q_heads < 1 || p->kv_heads < 1 || p->tokens < 1 || p->q_heads % p->kv_heads)
    return set_error(MIKV_ERR_INVALID_ARG, "%s: bad sizes", who);
  const int G = p->q_heads / p->kv_heads;
  if (G != 1 && G != 2 && G != 4 && G != 8)
    return set_error(MIKV_ERR_UNSUPPORTED, "%s: query heads per KV head must be 1, 2, 4 or 8", who);
  if (p->head_dim != kHeadDim) return set_error(MIKV_ERR_UNSUPPORTED, "%s: head_dim must be %d", who, kHeadDim);
  if (!(p->scale > 0.0f) || p->scale == kInf) return set_error(MIKV_ERR_INVALID_ARG, "%s: scale must be > 0", who);
  if (p->tokens > 1 << 30) return set_error(MIKV_ERR_UNSUPPORTED, "%s: over 2^30 tokens", who);
  // blocks of 64 rows at most, rounded up to whole groups and runs
  if ((int64_t)(p->batch * (int64_t)p->q_heads + 8 * G) * ((p->tokens + 63) / 64 + 32) > (int64_t)1 << 22 << 9)
    return set_error(MIKV_ERR_UNSUPPORTED, "%s: too many blocks", who);
  if (int e = check_rows(who, "q", p->q, p->q_stride)) return e;
  if (int e = check_rows(who, "k", p->k, p->k_stride)) return e;
  if (r) {
    if (int e = check_cap(r->cap, p->scale, who)) return e;
    if (r->window < 0) return set_error(MIKV_ERR_INVALID_ARG, "%s: window must be >= 0", who);
    if (((uintptr_t)r->slopes | (uintptr_t)r->begin | (uintptr_t)r->end) % 4)
      return set_error(MIKV_ERR_INVALID_ARG, "%s: misaligned rules", who);
  }
  return MIKV_OK;
}

// log2 units: s log2(e) = scale' d, or cap' tanh(scale' d) = d P(d^2) up to poly.limit
template <class Args>
void score_scales(float scale, float cap, Args &A) {
  A.cap = cap * kLog2e;
  A.scale = cap > 0.0f ? scale / cap : scale * kLog2e;
  if (cap > 0.0f) {
    const double a = (double)scale / cap, z = a * a, c = (double)scale * kLog2e;
    A.poly.c0 = (float)c;
    A.poly.c1 = (float)(c * z * kTanhQ0);
    A.poly.c2 = (float)(c * z * z * kTanhQ1);
    A.poly.c3 = (float)(c * z * z * z * kTanhQ2);
    A.poly.c4 = (float)(c * z * z * z * z * kTanhQ3);
    A.poly.limit = (float)(kTanhSmall / a);
  }
}

unsigned grid_blocks(int units, int per_unit, int run) {
  return (unsigned)(8 * ((units + 7) / 8) * (((int64_t)per_unit + run - 1) / run * run));
}

// XCDs that a unit's blocks go to: the fewest that leave the eight evenly filled to an
// eighth, so one unless there are few units.
int unit_parts(int64_t units) {
  int parts = 1;
  while (parts < 8 && ((units * parts + 7) / 8 * 8 - units * parts) * 8 > units * parts) parts *= 2;
  return parts;
}

template <class T>
void copy3(T d[3], const T s[3]) { d[0] = s[0], d[1] = s[1], d[2] = s[2]; }

template <int NW>
void launch_attention(PromptArgs &A, int G, bool cap, bool bias, hipStream_t st) {
  const int hw = std::min(G, NW), rows = kWaveQueries * (NW / hw), per_unit = (A.T + rows - 1) / rows * (G / hw);
  A.nblk = (A.T + rows - 1) / rows;
  A.parts = unit_parts(A.units);
  const int per_part = (per_unit + A.parts - 1) / A.parts;
  A.run = (int)std::min<int64_t>((int64_t)A.units * per_unit >= 4096 ? 32 : 4, per_part);
  const dim3 grid(grid_blocks(A.units * A.parts, per_part, A.run));
  auto kernel = cap ? (bias ? prompt_attention_kernel<true, true, NW> : prompt_attention_kernel<true, false, NW>)
                    : (bias ? prompt_attention_kernel<false, true, NW> : prompt_attention_kernel<false, false, NW>);
  hipLaunchKernelGGL(kernel, grid, dim3(64 * NW), 0, st, A);
}

template <int WS>
void launch_colsum(const SumArgs &A, dim3 grid, hipStream_t st) {
  const bool cap = A.cap > 0.0f, bias = A.slopes != nullptr;
  auto kernel = cap ? (bias ? prompt_colsum_kernel<WS, true, true> : prompt_colsum_kernel<WS, true, false>)
                    : (bias ? prompt_colsum_kernel<WS, false, true> : prompt_colsum_kernel<WS, false, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, A);
}

}  // namespace

}  // namespace mikv

using namespace mikv;

extern "C" int mikv_prompt_attention(const mikv_prompt *p, const mikv_score_rules *rules, uint16_t *out,
                                     const int64_t out_stride[3], float *lse, void *stream) {
  const char *who = "mikv_prompt_attention";
  if (int e = check_prompt(who, p, rules)) return e;
  if (int e = check_rows(who, "v", p->v, p->v_stride)) return e;
  if (!out_stride) return set_error(MIKV_ERR_INVALID_ARG, "%s: out_stride is NULL", who);
  if (int e = check_rows(who, "out", out, out_stride)) return e;
  if ((p->batch > 1 && !out_stride[0]) || (p->q_heads > 1 && !out_stride[1]) || (p->tokens > 1 && !out_stride[2]))
    return set_error(MIKV_ERR_INVALID_ARG, "%s: the output's rows share memory (stride 0)", who);
  if ((uintptr_t)lse % 4) return set_error(MIKV_ERR_INVALID_ARG, "%s: misaligned lse", who);
  PromptArgs A{};
  A.q = p->q, A.k = p->k, A.v = p->v, A.out = out, A.lse = lse;
  copy3(A.qs, p->q_stride), copy3(A.ks, p->k_stride), copy3(A.vs, p->v_stride), copy3(A.os, out_stride);
  if (rules) A.slopes = rules->slopes, A.begin = rules->begin, A.end = rules->end, A.window = rules->window;
  A.q_heads = p->q_heads, A.kv_heads = p->kv_heads, A.T = p->tokens;
  A.units = p->batch * p->kv_heads;
  const int G = p->q_heads / p->kv_heads;
  score_scales(p->scale, rules ? rules->cap : 0.0f, A);
  const bool cap = A.cap > 0.0f, bias = A.slopes != nullptr;
  // Waves per block: eight share each K and V row, four (two blocks to a CU) leave a
  // shorter tail and wait less for each other.  Eight only for long prompts, or groups that
  // fill a block with few query tiles, while there are blocks enough.  Measured
  // (us, eight -> four): 1 x 32/8 heads x 4096 146 -> 166, 2 x 32 x 8192 1130 -> 1206,
  // packed documents 16 x 32/8 x 2011 (tiles forwards) 330 -> 340, but 2 x 40 x 1531 90 -> 77,
  // 8 x 32 x 2048 397 -> 397, 1 x 8 x 8192 202 -> 187; under a cap or a bias alike (with a bias
  // 1 x 32/8 x 4096 143 -> 162, 2 x 40 x 1531 96 -> 83).
  const int64_t blocks = (int64_t)p->batch * p->q_heads * ((p->tokens + 255) / 256);
  if (p->tokens >= 4096 ? blocks >= 512 : G >= 4 && blocks >= 1024)
    launch_attention<8>(A, G, cap, bias, (hipStream_t)stream);
  else
    launch_attention<4>(A, G, cap, bias, (hipStream_t)stream);
  return check_launch(who);
}

// Workspace: the intervals of every 32 queries, then, where heads share a KV head,
// every query head's sums.
static size_t spans_bytes(int32_t batch, int32_t tokens) { return (size_t)batch * (((size_t)tokens + 31) / 32) * sizeof(int4); }

extern "C" size_t mikv_prompt_importance_workspace_size(int32_t batch, int32_t q_heads, int32_t kv_heads, int32_t tokens) {
  if (batch < 1 || q_heads < 1 || kv_heads < 1 || tokens < 1) return 0;
  return spans_bytes(batch, tokens) + (q_heads > kv_heads ? (size_t)batch * q_heads * tokens * sizeof(float) : 0);
}

extern "C" int mikv_prompt_importance(const mikv_prompt *p, const mikv_score_rules *rules, const float *lse, float *scores,
                                      void *ws, size_t ws_bytes, void *stream) {
  const char *who = "mikv_prompt_importance";
  if (int e = check_prompt(who, p, rules)) return e;
  if (!lse || !scores || ((uintptr_t)lse | (uintptr_t)scores) % 4)
    return set_error(MIKV_ERR_INVALID_ARG, "%s: NULL or misaligned lse or scores", who);
  if (!ws || ws_bytes < mikv_prompt_importance_workspace_size(p->batch, p->q_heads, p->kv_heads, p->tokens))
    return set_error(MIKV_ERR_CAPACITY, "%s: workspace too small", who);
  if ((uintptr_t)ws % 16) return set_error(MIKV_ERR_INVALID_ARG, "%s: workspace must be 16-byte aligned", who);
  hipStream_t st = (hipStream_t)stream;
  const int G = p->q_heads / p->kv_heads;
  SumArgs A{};
  A.q = p->q, A.k = p->k, A.lse = lse;
  A.sums = G > 1 ? (float *)((char *)ws + spans_bytes(p->batch, p->tokens)) : scores;
  copy3(A.qs, p->q_stride), copy3(A.ks, p->k_stride);
  if (rules) A.slopes = rules->slopes, A.begin = rules->begin, A.end = rules->end, A.window = rules->window;
  A.q_heads = p->q_heads, A.kv_heads = p->kv_heads, A.T = p->tokens;
  A.units = p->batch * p->kv_heads;
  score_scales(p->scale, rules ? rules->cap : 0.0f, A);
  const bool spans = A.begin || A.end || A.window;
  if (spans) {
    const int nsub = (p->tokens + 31) / 32;
    A.spans = (const int4 *)ws;
    for (int b = 0; b < p->batch; b += 65535)
      hipLaunchKernelGGL(query_spans_kernel, dim3((p->tokens + 63) / 64, std::min(65535, p->batch - b)), dim3(64), 0, st,
                         A.begin ? A.begin + (int64_t)b * p->tokens : nullptr, A.end ? A.end + (int64_t)b * p->tokens : nullptr,
                         A.window, p->tokens, nsub, (int4 *)ws + (int64_t)b * nsub);
  }
  // Waves on the same keys, by the blocks of 256 keys (two fit a CU, 512 the chip): as for
  // the causal scores (plan_pass), fewer keys per block only while the grid leaves CUs
  // idle.  Measured with 1 / 2 / 4 waves on the same keys, us: 8 x 32/8 x 4096 (4096
  // blocks) 705 / 864 / 1147, under documents and a cap 406 / 484 / 664; 1 x 40 x 1531
  // (240) 53 / 38 / 44; 1 x 32 x 512 (64) 25 / 19 / 15.
  const int64_t n1 = (int64_t)A.units * G * ((p->tokens + 255) / 256);
  const int share = n1 >= 768 ? 1 : n1 >= 192 ? 2 : 4;
  const int keys = kWaveRows * 4 / share;
  A.nblk = (p->tokens + keys - 1) / keys;
  A.parts = unit_parts(A.units);
  const int per_part = (A.nblk * G + A.parts - 1) / A.parts;
  // Runs of one key block's heads, which read the same keys: longer ones put long blocks at
  // the grid's end (8 x 32 x 2048: runs of one 205 us, of 32 267; 2 x 32 x 8192 630 and 701;
  // packed documents 8 x 32/8 x 4096: of one 517, of four 412, of 32 427).
  A.run = std::min(G, per_part);
  const dim3 grid(grid_blocks(A.units * A.parts, per_part, A.run));
  if (share == 1)
    launch_colsum<1>(A, grid, st);
  else if (share == 2)
    launch_colsum<2>(A, grid, st);
  else
    launch_colsum<4>(A, grid, st);
  if (G > 1)
    hipLaunchKernelGGL(sum_heads_kernel, dim3((p->tokens + 255) / 256, std::min(65535, A.units), (A.units + 65534) / 65535),
                       dim3(256), 0, st, (const float *)A.sums, A.units, G, p->tokens, scores);
  return check_launch(who);
}
