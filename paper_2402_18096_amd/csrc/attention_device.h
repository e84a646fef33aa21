// Decode-step attention over the mixed-precision cache (Section 3.4, Fig. 3
// left) and the importance update (the H2O accumulated-attention score).
//
// Split-K over the sequence: every block takes one contiguous chunk of one
// pool of one (sequence, KV head) -- chunks are homogeneous in precision
// (the pools are grouped by precision, which permutation invariance allows)
// and sized by bytes, so fp16/INT8 and INT2/INT4 chunks cost about the same.
// A block serves all G query heads of the KV group, so GQA loads K/V once.
//
// One wave per chunk (many small work units keep every CU streaming).
// Lanes: LPT = 128/CPL lanes per token, each owning CPL channels (CPL = 32;
// 16 from four query heads per KV head and for fp16 importance rows, whose
// lanes hold two spread 16-byte pieces so a token's lanes read whole
// 128-byte lines; 8 at eight query heads per KV head); a wave covers
// 64/LPT tokens per tile and UNROLL tiles per iteration.  Rows are read
// through buffer descriptors spanning the head's occupied slots (reads past
// them return zero and are masked), contiguous across the lanes of a tile:
// plainly for the cache's resident share (kept in the last-level cache from
// one step to the next), non-temporally for the rest.
//
// Inner loop, with every code c in [0, 2^N) of a group with scale alpha and
// zero beta (Eq. 1, decoded value alpha*c + beta):
//   score:  q . k = alpha * sum_c q_c code_c + beta * sum_c q_c
//   value:  e * v = (e*alpha) * code + e*beta, the e*beta part summed apart.
// Codes are turned into fp16 operands with one AND per two codes: a code c
// placed in the mantissa bits of a zero-exponent half is the fp16 subnormal
// c * 2^(s-24), s the code's bit offset inside the half (codes never reach
// the exponent bits; offsets 10..15 are shifted down first).  Products with
// such halves are exact in fp32, the 2^(s-24) factors are folded into the
// query (key side, v_dot2_f32_f16) and into the final sums (value side,
// fp32 fma with an fp16 operand).  fp16 rows are used as stored.
//
// Softmax: the running maximum is wave-uniform and only raised when a score
// exceeds it by more than 2^8 in the exponential (checked with a ballot), so
// the common tile needs no cross-lane max.  Scores are kept in log2 units.
// The partial phase writes per-chunk (max, sum, value-sum) records and the
// scores; the finalize phase merges the records exactly, turns scores into
// probabilities and optionally adds them to the importance scores.
#ifndef MIKV_ATTENTION_DEVICE_H
#define MIKV_ATTENTION_DEVICE_H

#include <type_traits>

#include "../../include/mikv_layer.h"
#include "append_device.h"
#include "mikv_internal.h"

namespace mikv {

// Score rules of the decode attention (RULES kernels): the scale of a dot product
// that tanh takes and the cap in log2 units (cap 0: none), slopes of the bias by
// distance, first visible position per sequence.
struct RuleArgs {
  float cap_scale, cap;
  const float *slopes;
  const int32_t *begin;
  int last;    // position of the query
  int window;  // last positions seen (0: all)
};

struct AttnArgs {
  const uint8_t *hi_k, *hi_v;
  const uint32_t *hi_kp, *hi_vp;
  const int32_t *n_hi;
  const uint8_t *lo_k, *lo_v;
  const uint32_t *lo_kp, *lo_vp;
  const int32_t *n_lo;
  const uint16_t *q;
  const float *balance;
  float scale;
  float *scores_hi, *scores_lo;  // [B*Hq, cap] scores in log2 units (nullable)
  float *partials;               // [B*Hq, nc_hi + nc_lo, kRec]
  float *probs_hi, *probs_lo;    // outputs (nullable)
  float *acc;                    // hi_acc when accumulating (nullable)
  float *out;                    // [B*Hq, 128]
  int cap_hi, cap_lo, group, q_heads, kv_heads;
  int chunk_hi, chunk_lo, nc_hi, nc_lo, nc_first;
  // Decode step: the new token is appended by the partial phase (app.k
  // non-NULL) and n_hi does not count it until the re-rank writes it.
  AppendArgs app;
  int hi_pending;
  int pool_major;  // dispatch every importance-pool chunk first (fp16 importance pools under GQA)
  int res_hi, res_lo;  // heads [0, res) of each pool are read plainly, the others streamed
  int order;       // 0: the grid order below; 1: heads reversed; 2: the whole grid reversed
  // per-channel retained keys (key_block 64): (alpha, beta) words
  // [NH, n_kblk, 128] per key block, found through the token's position
  const uint32_t *lo_kb;
  const int32_t *lo_pos;
  int n_kblk;
  const int32_t *hi_pos;
  RuleArgs rules;
};

// The partial phase under score rules (attention_rules.hip).
void launch_partial_rules(const AttnArgs &A, const mikv_cache *c, bool lean, dim3 grid, hipStream_t st);

namespace {

constexpr int kBlock = 256;        // finalize / importance kernels
constexpr int kWaves = 1;          // the partial kernel runs one wave per chunk
// Chunk record per query head and chunk: max, sum, the pool's token count
// as the partial phase saw it (int32 bits), a pad word, value sum[128]
// (kept 16-byte aligned for vector loads).
constexpr int kRecN = 2;
constexpr int kRecO = 4;
constexpr int kRec = kRecO + kHeadDim;
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLog2e = 1.4426950408889634f;
// The scores (written by the partial kernel into the probability arrays)
// and the probabilities that replace them are each touched once per step:
// they are written and read with non-temporal hints, so that this traffic
// does not push the cache rows out of the last-level cache, from which the
// next step reads part of them again (measured at the Mistral shape: 75 ->
// 70 us per attention launch, 97 -> 92 us per step).
constexpr float kLazy = 8.0f;       // raise the running max only past this (log2 units)
constexpr int kMaxChunk = 1024;     // tokens per chunk at most (the chunk's scores are held in LDS)
// Tokens per chunk at most for G query heads per KV head: the chunk's
// scores (G x chunk fp32) stay within 8 KiB of LDS, so LDS does not bound
// the waves per CU below what the registers allow.
__host__ __device__ constexpr int max_chunk(int G) { return G <= 2 ? kMaxChunk : 2048 / G; }

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));


// Importance-pool tokens of head h, the pending new token included.
__device__ inline int hi_count(const AttnArgs &A, int h) {
  const int n = A.n_hi[h];
  return n + (A.hi_pending && n < A.cap_hi ? 1 : 0);
}

// The score of one token in log2 units under the rules, from its dot product's
// score without them (`plain`, log2 units) or the argument of tanh (`arg`).
__device__ inline float rule_score(const RuleArgs &R, float plain, float arg, float slope2, int pos) {
  const float s = R.cap > 0.0f ? R.cap * tanh_fine(arg) : plain;
  return fmaf(-slope2, fabsf((float)(R.last - pos)), s);
}

// First position that sequence b sees.
__device__ inline int rule_begin(const RuleArgs &R, int b) {
  const int first = R.window > 0 ? R.last + 1 - min(R.window, R.last + 1) : 0;
  return R.begin ? max(first, __builtin_amdgcn_readfirstlane(R.begin[b])) : first;
}
// Whether a rule needs the tokens' positions; otherwise their descriptor is
// empty and every position reads as 0.
__device__ inline bool rule_positions(const RuleArgs &R) { return R.slopes || R.begin || R.window > 0; }

// ---------------------------------------------------------------------------
// Packed-row formats.  A lane's CPL channels are held as NP = CPL/2 fp16
// pairs; pair p holds lane-local channels lo(p) and hi(p), scaled by
// 2^(cls(p) - 24) for codes (exact fp16 subnormals), or the stored fp16
// values for BITS == 16.
// ---------------------------------------------------------------------------
// FINE: 2-, 3- and 4-bit codes moved up to mantissa bits 6-9 (classes 6 and 8).
// The dot products multiply the deepest subnormals at reduced precision (scores
// of 2-bit keys 3e-6 off against 2e-7 with FINE); a shift more for every four codes.
template <int BITS, bool FINE = false>
struct Fmt {
  static constexpr bool kQuant = BITS != 16;
  __host__ __device__ static constexpr int lo(int p) {
    return BITS == 16 || BITS == 3 ? 2 * p
         : BITS == 8  ? 4 * (p / 2) + p % 2
         : BITS == 4  ? 8 * (p / 4) + p % 4
                      : 16 * (p / 8) + p % 8;
  }
  __host__ __device__ static constexpr int hi(int p) {
    return BITS == 16 || BITS == 3 ? 2 * p + 1 : lo(p) + (BITS == 8 ? 2 : BITS == 4 ? 4 : 8);
  }
  __host__ __device__ static constexpr int cls(int p) {
    if (FINE) return BITS == 2 ? 6 + 2 * (p % 2) : BITS == 3 || BITS == 4 ? 6 : 0;
    return BITS == 4 ? 4 * (p % 2) : BITS == 2 ? 2 * (p % 4) : 0;
  }
  // largest and smallest class
  static constexpr int kMaxCls = FINE ? (BITS == 2 ? 8 : BITS == 3 || BITS == 4 ? 6 : 0) : BITS == 2 ? 6 : BITS == 4 ? 4 : 0;
  static constexpr int kMinCls = FINE && BITS <= 4 ? 6 : 0;
  template <int CPL>
  __device__ static inline void unpack(const uint32_t *raw, uint32_t *out) {
    if constexpr (BITS == 16) {
#pragma unroll
      for (int j = 0; j < CPL / 2; ++j) out[j] = raw[j];
    } else if constexpr (BITS == 3) {
      // 3-bit codes straddle bytes and words: each pair (channels 2j,
      // 2j+1, bits 6j .. 6j+5 of the lane's 3 CPL bits, which start at bit
      // 0 of raw[0]) is extracted from the 64-bit window that holds it into
      // the low bits of the two halves
      constexpr int KW = CPL == 32 ? 3 : 2;
#pragma unroll
      for (int j = 0; j < CPL / 2; ++j) {
        const int bit = 6 * j, wi = bit / 32, sh = bit % 32;
        const uint64_t win = ((uint64_t)(wi + 1 < KW ? raw[wi + 1] : 0u) << 32) | raw[wi];
        if constexpr (FINE) {
          const uint32_t x = (uint32_t)(sh >= 6 ? win >> (sh - 6) : win << (6 - sh));
          out[j] = (x & 0x1c0u) | ((x << 13) & 0x01c00000u);
        } else {
          const uint32_t x = (uint32_t)(win >> sh);
          out[j] = (x & 7u) | (((x >> 3) & 7u) << 16);
        }
      }
    } else if constexpr (BITS == 8) {
#pragma unroll
      for (int j = 0; j < CPL / 4; ++j) {
        out[2 * j] = raw[j] & 0x00ff00ffu;
        out[2 * j + 1] = (raw[j] >> 8) & 0x00ff00ffu;
      }
    } else if constexpr (FINE && BITS == 4) {
#pragma unroll
      for (int j = 0; j < CPL / 8; ++j) {
        const uint32_t x = raw[j];
        out[4 * j] = (x << 6) & 0x03c003c0u;
        out[4 * j + 1] = (x << 2) & 0x03c003c0u;
        out[4 * j + 2] = (x >> 2) & 0x03c003c0u;
        out[4 * j + 3] = (x >> 6) & 0x03c003c0u;
      }
    } else if constexpr (FINE) {
#pragma unroll
      for (int j = 0; j < CPL / 16; ++j) {
        const uint32_t x = raw[j], s[4] = {x << 6, x << 2, x >> 2, x >> 6};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          out[8 * j + 2 * k] = s[k] & 0x00c000c0u;
          out[8 * j + 2 * k + 1] = s[k] & 0x03000300u;
        }
      }
    } else if constexpr (BITS == 4) {
#pragma unroll
      for (int j = 0; j < CPL / 8; ++j) {
        const uint32_t x = raw[j], y = x >> 8;
        out[4 * j] = x & 0x000f000fu;
        out[4 * j + 1] = x & 0x00f000f0u;
        out[4 * j + 2] = y & 0x000f000fu;
        out[4 * j + 3] = y & 0x00f000f0u;
      }
    } else {
#pragma unroll
      for (int j = 0; j < CPL / 16; ++j) {
        const uint32_t x = raw[j], y = x >> 8;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          out[8 * j + k] = x & (0x00030003u << (2 * k));
          out[8 * j + 4 + k] = y & (0x00030003u << (2 * k));
        }
      }
    }
  }
};

__device__ inline half2_t as_h2(uint32_t u) { return __builtin_bit_cast(half2_t, u); }

// Codes enter the dot products as fp16 subnormals code * 2^(cls - 24), so
// the query channel paired with a code of class cls is scaled by 2^-cls.
// Scaled down, a small query channel would itself become an fp16 subnormal
// and lose bits (and the matrix cores handle subnormal operands at reduced
// precision), so the query is instead scaled by 2^(shift - cls) with shift
// = the format's largest cls: never below 1, exact in fp16.  A wave whose
// largest |q_hat| would overflow fp16 that way keeps shift 0.  The shift is
// undone in the score scale (wave-uniform).
// (smallest class MINCLS: the largest factor is 2^(MAXCLS - MINCLS).)
template <int MAXCLS, int MINCLS = 0>
__device__ inline int query_shift(float qmax_lane) {
  if constexpr (MAXCLS == MINCLS) {
    return MAXCLS;
  } else {
    const float m = wave_max(qmax_lane);
    return m * (float)(1 << (MAXCLS - MINCLS)) < 60000.0f ? MAXCLS : MINCLS;
  }
}

// Sum over the LPT consecutive lanes of a token (LPT = 4, 8 or 16).
template <int LPT>
__device__ inline float token_sum(float v) {
  v += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0xB1, 0xF, 0xF, true));
  v += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x4E, 0xF, 0xF, true));
  if constexpr (LPT >= 8)  // other quad of the half-row
    v += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x141, 0xF, 0xF, true));
  if constexpr (LPT == 16)  // other half of the row
    v += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x140, 0xF, 0xF, true));
  return v;
}

// token_sum of G values at once that leaves each lane only the sum of value
// part % G: while a bit of `part` numbers values, a lane keeps the half that its bit names
// and gives the other half away.  v[0] is the sum.
template <int LPT, int G, int SPAN = LPT / 2, int N = G>
__device__ inline float token_sum_own(float (&v)[G]) {
  auto other = [](float x) { return dpp_mov<SPAN == 8 ? 0x140 : SPAN == 4 ? 0x141 : SPAN == 2 ? 0x4E : 0xB1>(x); };
  if constexpr (SPAN == 0) {
    return v[0];
  } else if constexpr (SPAN < G) {
    const bool up = lanes_with<SPAN>();
#pragma unroll
    for (int k = 0; k < N / 2; ++k) v[k] = (up ? v[k + N / 2] : v[k]) + other(up ? v[k] : v[k + N / 2]);
    return token_sum_own<LPT, G, SPAN / 2, N / 2>(v);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += other(v[k]);
    return token_sum_own<LPT, G, SPAN / 2, N>(v);
  }
}

// The other way: every lane gets the G values that the lanes part % G of its token hold.
template <int G>
__device__ inline void token_share(float own, float (&v)[G]) {
  if constexpr (G == 1) {
    v[0] = own;
  } else if constexpr (G == 2) {
    v[0] = dpp_mov<0xA0>(own);
    v[1] = dpp_mov<0xF5>(own);
  } else {
    v[0] = dpp_mov<0x00>(own);
    v[1] = dpp_mov<0x55>(own);
    v[2] = dpp_mov<0xAA>(own);
    v[3] = dpp_mov<0xFF>(own);
    if constexpr (G == 8) {
      const bool up = lanes_with<4>();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = dpp_mov<0x141>(v[i]);  // the other quad of the half-row
        v[i + 4] = up ? v[i] : x;
        v[i] = up ? x : v[i];
      }
    }
  }
}

// Sum over the 64/LPT lanes that hold the same `part` (same channels,
// different tokens): rotations inside each 16-lane row, shuffles across rows.
template <int LPT>
__device__ inline float sum_token_lanes(float v) {
  if constexpr (LPT == 4) {
    v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x124, 0xF, 0xF, false));
    v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x128, 0xF, 0xF, false));
  } else if constexpr (LPT == 8) {
    v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x128, 0xF, 0xF, false));
  }  // LPT 16: one token per row
  v += __shfl_xor(v, 16, 64);
  v += __shfl_xor(v, 32, 64);
  return v;
}

// A reduction over the lanes of the same number modulo G (1, 2, 4 or 8), in every lane.
template <int G, class Op>
__device__ inline float over_lanes(float v, Op op) {
  if constexpr (G <= 1) v = op(v, dpp_mov<0xB1>(v));
  if constexpr (G <= 2) v = op(v, dpp_mov<0x4E>(v));
  if constexpr (G <= 4) v = op(v, dpp_mov<0x124>(v));
  v = op(v, dpp_mov<0x128>(v));
  return with_half(with_row(v, op), op);
}

// A 3-bit lane segment of 16 (8) channels is 48 (24) bits: two dwords are
// loaded from the dword that holds its first bit and shifted (seg_shift) so
// that the segment starts at bit 0.
template <int BITS, int CPL>
struct Rows {
  static constexpr int KW = BITS == 16 ? CPL / 2 : BITS == 3 && CPL <= 16 ? 2 : CPL * BITS / 32;  // raw dwords per segment
  uint32_t k[KW], v[KW];
  uint32_t kp, vp;
  uint32_t pos;  // the token's position (RULES)
};

typedef __amdgpu_buffer_rsrc_t rsrc_t;
// Cache-policy bits of the cache-row loads: streamed rows are read
// non-temporally (the nt bit), the rest plainly; see attn_partial_kernel.
constexpr int kStreamPolicy = 2;
constexpr int kRsrcFlags = 0x00020000;  // raw (untyped) buffer, gfx9 descriptor word 3

// A buffer resource over `bytes` bytes at `base`: loads at offsets past the
// end return zero (so reading past the occupied slots of a pool is safe).
__device__ inline rsrc_t make_rsrc(const void *base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), (short)0, (int)bytes, kRsrcFlags);
}

// Load one token's row segments (this lane's channels) and group params at
// byte offsets `orow` (rows) and `opar` (params) of the head's pools.
// WHICH: 1 the key segment and its group parameters, 2 the value's, 3 both.
// PIECE: bytes between the lane's 16-byte pieces of a row; CPOL: the
// loads' cache-policy bits.
template <int BITS, int CPL, int WHICH = 3, int PIECE = 16, int CPOL = 0>
__device__ inline void load_seg_rows(Rows<BITS, CPL> &r, rsrc_t rk, rsrc_t rv, rsrc_t rkp, rsrc_t rvp, uint32_t orow,
                                     uint32_t opar, uint32_t okp) {
  constexpr int KW = Rows<BITS, CPL>::KW;
  constexpr bool LK = (WHICH & 1) != 0, LV = (WHICH & 2) != 0;
  if constexpr (KW >= 4) {
#pragma unroll
    for (int i = 0; i < KW / 4; ++i) {
      if constexpr (LK) {
        auto a = __builtin_amdgcn_raw_buffer_load_b128(rk, orow + PIECE * i, 0, CPOL);
#pragma unroll
        for (int j = 0; j < 4; ++j) r.k[4 * i + j] = a[j];
      }
      if constexpr (LV) {
        auto b = __builtin_amdgcn_raw_buffer_load_b128(rv, orow + PIECE * i, 0, CPOL);
#pragma unroll
        for (int j = 0; j < 4; ++j) r.v[4 * i + j] = b[j];
      }
    }
  } else if constexpr (KW == 3) {
    if constexpr (LK) {
      auto a = __builtin_amdgcn_raw_buffer_load_b96(rk, orow, 0, CPOL);
      r.k[0] = a[0]; r.k[1] = a[1]; r.k[2] = a[2];
    }
    if constexpr (LV) {
      auto b = __builtin_amdgcn_raw_buffer_load_b96(rv, orow, 0, CPOL);
      r.v[0] = b[0]; r.v[1] = b[1]; r.v[2] = b[2];
    }
  } else if constexpr (KW == 2) {
    if constexpr (LK) {
      auto a = __builtin_amdgcn_raw_buffer_load_b64(rk, orow, 0, CPOL);
      r.k[0] = a[0]; r.k[1] = a[1];
    }
    if constexpr (LV) {
      auto b = __builtin_amdgcn_raw_buffer_load_b64(rv, orow, 0, CPOL);
      r.v[0] = b[0]; r.v[1] = b[1];
    }
  } else {
    if constexpr (LK) r.k[0] = __builtin_amdgcn_raw_buffer_load_b32(rk, orow, 0, CPOL);
    if constexpr (LV) r.v[0] = __builtin_amdgcn_raw_buffer_load_b32(rv, orow, 0, CPOL);
  }
  if constexpr (BITS != 16) {
    if constexpr (LK) r.kp = __builtin_amdgcn_raw_buffer_load_b32(rkp, okp, 0, CPOL);
    if constexpr (LV) r.vp = __builtin_amdgcn_raw_buffer_load_b32(rvp, opar, 0, CPOL);
  }
}

// RULES: the iterations [lo, hi) of PER tokens outside of which slots [start, end) of a
// pool hold no token from position `begin` on.  The pools keep the prompt's order, so
// whole chunks are left out of a windowed or padded cache; looking costs a trip to memory, so
// only where at least a quarter of the positions is hidden (16 x 32/8 x 16384, fp16 over
// INT2, the last 4096 positions: 83 us without it, 60 with).
template <int PER>
__device__ inline void visible_range(const RuleArgs &R, rsrc_t rpos, int begin, int start, int end, int &lo, int &hi) {
  if (end <= start || begin == 0 || (int64_t)begin * 4 < R.last) return;  // (an empty chunk ends before it starts)
  int first = end, last = start - 1;
  for (int s = start + (int)(threadIdx.x & 63); s < end; s += 64)
    if ((int)__builtin_amdgcn_raw_buffer_load_b32(rpos, (uint32_t)s * 4u, 0, 0) >= begin) {
      first = min(first, s);
      last = s;
    }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    first = min(first, __shfl_xor(first, o, 64));
    last = max(last, __shfl_xor(last, o, 64));
  }
  first = __builtin_amdgcn_readfirstlane(first);
  last = __builtin_amdgcn_readfirstlane(last);
  lo = last < first ? 0 : (first - start) / PER;
  hi = last < first ? 0 : (last - start) / PER + 1;
}

// KPC: retained keys quantized per channel over 64-position blocks
// (Appendix C).  The key's "parameter" word is then its position; a lane
// keeps q_c * alpha_c (times the code class factor) and sum_c q_c beta_c for
// the block of its current token and refreshes them when the block changes.
// RULES: scores under A.rules.  A token's position comes with its key; one that is
// hidden gets a score of -inf and adds nothing, whatever its row holds.  The lanes of
// a token share out its G scores (lane part % G keeps one): a rule and an
// exponential per lane, not G of them (16 x 32/8 x 8192, fp16 over INT4, under a cap:
// every lane scoring every head 104 us, this 78, and 78 without rules).  Chunks run
// backwards, so that under a bias by distance the first scores are the largest and the
// running maximum stays (16 x 32/8 x 16384, fp16 over INT2: forwards 98 us, both 84).
template <int BITS, int G, int CPL, bool SPLITQ, int UNROLL, int PREFETCH, bool KPC = false, bool STREAM = false, bool RULES = false>
__device__ void attn_chunk(const AttnArgs &A, int h, int chunk, int rec_chunk, bool is_hi, float *s_lds) {
  using F = Fmt<BITS>;
  using FK = Fmt<BITS, RULES && !KPC>;  // keys (the per-channel ones enter fp32 FMAs, which are exact)
  constexpr int LPT = kHeadDim / CPL, TPW = 64 / LPT, NP = CPL / 2;
  constexpr bool Q = F::kQuant;
  constexpr int S = RULES ? 1 : G;  // scores, maxima and sums a lane keeps
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int part = lane % LPT, tsub = lane / LPT;
  const int b = h / A.kv_heads, kvh = h % A.kv_heads;
  const int qh0 = b * A.q_heads + kvh * G;

  const int cap = is_hi ? A.cap_hi : A.cap_lo;
  const int chunk_len = is_hi ? A.chunk_hi : A.chunk_lo;
  // The pool count comes through a vector load; make it provably
  // wave-uniform, so the buffer descriptors built from it live in scalar
  // registers (a value the compiler thinks divergent would wrap every load in
  // a per-lane loop).
  const int n_pool = __builtin_amdgcn_readfirstlane(is_hi ? hi_count(A, h) : A.n_lo[h]);
  const int start = chunk * chunk_len;
  const int end = min(start + chunk_len, n_pool);
  constexpr int64_t kRow = BITS == 16 ? kHeadDim * 2 : kHeadDim * BITS / 8;
  const int ng = kHeadDim / A.group;
  const uint8_t *kb = (is_hi ? A.hi_k : A.lo_k) + (int64_t)h * cap * kRow;
  const uint8_t *vb = (is_hi ? A.hi_v : A.lo_v) + (int64_t)h * cap * kRow;
  const uint32_t *kpb = Q ? (is_hi ? A.hi_kp : A.lo_kp) + (int64_t)h * cap * ng : nullptr;
  const uint32_t *vpb = Q ? (is_hi ? A.hi_vp : A.lo_vp) + (int64_t)h * cap * ng : nullptr;
  float *scores = is_hi ? A.scores_hi : A.scores_lo;
  const float s2scale = A.scale * kLog2e;

  // Query (Eq. 4: q / balance), as fp16 pairs matching the format's pairing,
  // each pair scaled by 2^(qshift - cls) (query_shift); with SPLITQ a second
  // fp16 pair carries the rounding remainder.  qsum24 = 2^(qshift - 24) * the
  // sum of the lane's query channels (fp32).
  float m2[S], l[S], bsum[G], o[G][CPL];
  const int own = RULES ? part % G : 0;  // this lane's query head
#pragma unroll
  for (int i = 0; i < S; ++i) {
    m2[i] = kNegInf;
    l[i] = 0.0f;
  }
#pragma unroll
  for (int i = 0; i < G; ++i) {
    bsum[i] = 0.0f;
#pragma unroll
    for (int c = 0; c < CPL; ++c) o[i][c] = 0.0f;
  }

  constexpr int kPerIter = kWaves * TPW * UNROLL;
  // chunks are whole iterations, at most max_chunk(G) tokens (multiples of
  // 128, or the shorter ones of make_plan from G = 4 on): an iteration never
  // runs past the LDS score buffer
  static_assert(128 % kPerIter == 0 && max_chunk(G) % 128 == 0, "iteration must divide 128 tokens");
  static_assert(G < 4 || kPerIter <= 16 || (BITS <= 4 && kPerIter <= 32), "and from G = 4 on the chunks of make_plan");
  constexpr int kSeg = Rows<BITS, CPL>::KW * 4;  // bytes loaded per lane's row segment
  // byte offset of the lane's segment in a row, and the bit shift that
  // aligns it (non-zero only for 3-bit segments of 48 or 24 bits, which
  // start inside a dword)
  constexpr bool kSeg3 = BITS == 3 && CPL <= 16;
  constexpr int kSeg3Bytes = 3 * CPL / 8;
  // fp16 rows are read spread: piece j of the lane (8 channels, 16 bytes)
  // holds channels 8 (part + LPT j) .. + 7, so each load of the LPT lanes of
  // a token covers whole 128-byte lines of its row, which streaming
  // (non-temporal) loads need to fetch every line once.  Other formats hold
  // CPL consecutive channels per lane.
  constexpr bool kSpread = BITS == 16;
  constexpr int kPiece = kSpread ? 16 * LPT : 16;
  auto chan8 = [&](int j) { return kSpread ? 8 * (part + LPT * j) : part * CPL + 8 * j; };  // first channel of piece j
  const uint32_t seg_off =
      kSeg3 ? 4u * (uint32_t)((kSeg3Bytes * part) / 4) : kSpread ? 16u * (uint32_t)part : (uint32_t)(part * kSeg);
  const int seg_shift = kSeg3 ? 8 * ((kSeg3Bytes * part) % 4) : 0;
  auto seg_words = [&](const uint32_t *raw, uint32_t *out) {
    if constexpr (kSeg3) {
      out[0] = __builtin_amdgcn_alignbit(raw[1], raw[0], seg_shift);
      out[1] = raw[1] >> seg_shift;
    } else {
#pragma unroll
      for (int i = 0; i < Rows<BITS, CPL>::KW; ++i) out[i] = raw[i];
    }
  };
  int n_iter = end > start ? (end - start + kPerIter - 1) / kPerIter : 0;
  const int first = start + wave * TPW * UNROLL + tsub;  // this lane's token in iteration 0, u = 0
  const int g_lane = (part * CPL) / A.group;
  // Buffer resources over this head's occupied slots; a lane's offset is
  // fixed per iteration and the unroll steps are immediate offsets.
  const rsrc_t rk = make_rsrc(kb, (uint32_t)n_pool * (uint32_t)kRow);
  const rsrc_t rv = make_rsrc(vb, (uint32_t)n_pool * (uint32_t)kRow);
  const rsrc_t rkp = KPC ? make_rsrc(A.lo_pos + (int64_t)h * cap, (uint32_t)n_pool * 4u)
                         : make_rsrc(Q ? (const void *)kpb : (const void *)kb, Q ? (uint32_t)n_pool * ng * 4u : 0u);
  const rsrc_t rvp = make_rsrc(Q ? (const void *)vpb : (const void *)vb, Q ? (uint32_t)n_pool * ng * 4u : 0u);
  const rsrc_t rpos = make_rsrc(RULES ? (const void *)((is_hi ? A.hi_pos : A.lo_pos) + (int64_t)h * cap) : (const void *)kb,
                                RULES && rule_positions(A.rules) ? (uint32_t)n_pool * 4u : 0u);
  int begin = 0, it_end = n_iter;  // first visible position; end of the iterations
  if constexpr (RULES) {
    begin = rule_begin(A.rules, b);
    int it_begin = 0;
    visible_range<kPerIter>(A.rules, rpos, begin, start, end, it_begin, it_end);
    if (it_end - it_begin < n_iter) {
      for (int i = 0; i < G; ++i)
        for (int j = lane; j < end - start; j += 64) s_lds[i * max_chunk(G) + j] = kNegInf;
    }
    n_iter = it_end - it_begin;
  }
  const uint32_t lane_tok = (uint32_t)(start + wave * TPW * UNROLL + tsub);
  const uint32_t off_row0 = lane_tok * (uint32_t)kRow + seg_off;
  const uint32_t off_par0 = (lane_tok * (uint32_t)ng + (uint32_t)g_lane) * 4u;
  const uint32_t off_kp0 = KPC ? lane_tok * 4u : off_par0;

  // With `live` false the loads go through empty descriptors: they return
  // zero without a memory access, so a load needs no branch around it.
  const rsrc_t r_none = make_rsrc(kb, 0u);
  auto load_part = [&](auto which, Rows<BITS, CPL>(&r)[UNROLL], int it, bool live = true) {
    if constexpr (RULES) it = it_end - 1 - it;
    const uint32_t orow = off_row0 + (uint32_t)(it * kPerIter) * (uint32_t)kRow;
    const uint32_t opar = off_par0 + (uint32_t)(it * kPerIter) * (uint32_t)ng * 4u;
    const uint32_t okp = KPC ? off_kp0 + (uint32_t)(it * kPerIter) * 4u : opar;
    const rsrc_t ak = live ? rk : r_none, av = live ? rv : r_none;
    const rsrc_t akp = live ? rkp : r_none, avp = live ? rvp : r_none;
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
      load_seg_rows<BITS, CPL, decltype(which)::value, kPiece, STREAM ? kStreamPolicy : 0>(r[u], ak, av, akp, avp, orow + (uint32_t)(u * TPW * kRow),
                                                       opar + (uint32_t)(u * TPW) * (uint32_t)ng * 4u,
                                                       KPC ? okp + (uint32_t)(u * TPW) * 4u
                                                           : opar + (uint32_t)(u * TPW) * (uint32_t)ng * 4u);
    if constexpr (RULES && (decltype(which)::value & 1) != 0) {
      const rsrc_t apos = live ? rpos : r_none;
#pragma unroll
      for (int u = 0; u < UNROLL; ++u)
        r[u].pos = __builtin_amdgcn_raw_buffer_load_b32(apos, (lane_tok + (uint32_t)(it * kPerIter + u * TPW)) * 4u, 0, STREAM ? kStreamPolicy : 0);
    }
  };
  auto load_it = [&](Rows<BITS, CPL>(&r)[UNROLL], int it) { load_part(std::integral_constant<int, 3>{}, r, it); };

  // The first iterations' rows do not depend on the query: issue them first.
  Rows<BITS, CPL> cur[UNROLL], n1[PREFETCH >= 1 ? UNROLL : 1], n2[PREFETCH >= 2 ? UNROLL : 1];
  if (n_iter > 0) load_it(cur, 0);
  if constexpr (PREFETCH >= 1) {
    if (n_iter > 1) load_it(n1, 1);
  }
  if constexpr (PREFETCH >= 2) {
    if (n_iter > 2) load_it(n2, 2);
  }

  // Every query (and balancer) word this lane needs is loaded with 16-byte
  // loads issued together, before any of them is used: the chunk's K/V
  // stream starts one memory round trip after the wave does.
  half2_t qh[G][NP], ql[G][SPLITQ ? NP : 1];
  float qsum24[G];  // 2^-24 * sum of the lane's query channels
  float qkeep[KPC ? G : 1][KPC ? CPL : 1];  // KPC: the lane's query channels (fp32)
  uint4 qraw[G][CPL / 8];
#pragma unroll
  for (int i = 0; i < G; ++i) {
    const uint16_t *qrow = A.q + (int64_t)(qh0 + i) * kHeadDim;
#pragma unroll
    for (int j = 0; j < CPL / 8; ++j) qraw[i][j] = *reinterpret_cast<const uint4 *>(qrow + chan8(j));
  }
  float bal[SPLITQ ? CPL : 1];
  if constexpr (SPLITQ) {
    const float *brow = A.balance + (int64_t)h * kHeadDim;
#pragma unroll
    for (int j = 0; j < CPL / 4; ++j) {
      const float4 v = *reinterpret_cast<const float4 *>(brow + chan8(j >> 1) + 4 * (j & 1));
      bal[4 * j] = v.x;
      bal[4 * j + 1] = v.y;
      bal[4 * j + 2] = v.z;
      bal[4 * j + 3] = v.w;
    }
  }
  constexpr int kMaxCls = FK::kMaxCls, kMinCls = FK::kMinCls;
  int qshift = 0;
  if constexpr (kMaxCls > 0 && !KPC) {
    // bound on |q_hat| over the wave: max |q| / min b
    uint32_t mb = 0;
#pragma unroll
    for (int i = 0; i < G; ++i)
#pragma unroll
      for (int j = 0; j < CPL / 8; ++j) {
        const uint32_t w[4] = {qraw[i][j].x, qraw[i][j].y, qraw[i][j].z, qraw[i][j].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) mb = max(mb, max(w[k] & 0x7fffu, (w[k] >> 16) & 0x7fffu));
      }
    float bound = f16_to_f32((uint16_t)mb);
    if constexpr (SPLITQ) {
      float bmin = bal[0];
#pragma unroll
      for (int c = 1; c < CPL; ++c) bmin = fminf(bmin, bal[c]);
      bound = bound / bmin;
    }
    qshift = query_shift<kMaxCls, kMinCls>(bound);
  }
  const float s2scale_q = Q ? __builtin_ldexpf(s2scale, 24 - qshift) : s2scale;
  float arg_scale = 0.0f, slope2 = 0.0f;
  if constexpr (RULES) {
    arg_scale = Q ? __builtin_ldexpf(A.rules.cap_scale, 24 - qshift) : A.rules.cap_scale;
    if (A.rules.slopes) slope2 = A.rules.slopes[kvh * G + own] * kLog2e;
  }
#pragma unroll
  for (int i = 0; i < G; ++i) {
    float qf[CPL];
#pragma unroll
    for (int j = 0; j < CPL / 8; ++j) {
      const uint32_t w[4] = {qraw[i][j].x, qraw[i][j].y, qraw[i][j].z, qraw[i][j].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        qf[8 * j + 2 * k] = f16_to_f32((uint16_t)(w[k] & 0xffffu));
        qf[8 * j + 2 * k + 1] = f16_to_f32((uint16_t)(w[k] >> 16));
      }
    }
    if constexpr (SPLITQ) {
#pragma unroll
      for (int c = 0; c < CPL; ++c) qf[c] = qf[c] / bal[c];
    }
    auto qhat = [&](int c) { return qf[c]; };
    if constexpr (KPC) {
#pragma unroll
      for (int c = 0; c < CPL; ++c) qkeep[i][c] = qf[c];
    }
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < CPL; ++c) s += qhat(c);
    qsum24[i] = __builtin_ldexpf(s, qshift - 24);
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const float sc = __builtin_ldexpf(1.0f, qshift - FK::cls(p));
      const float a = qhat(F::lo(p)) * sc, bb = qhat(F::hi(p)) * sc;
      const _Float16 ah = (_Float16)a, bh = (_Float16)bb;
      qh[i][p] = half2_t{ah, bh};
      if constexpr (SPLITQ) ql[i][p] = half2_t{(_Float16)(a - (float)ah), (_Float16)(bb - (float)bh)};
    }
  }

  // The chunk's scores stay in LDS (written by the lanes that hold them)
  // and go out in one burst after the loop: no global store is issued
  // between the loads of the stream (stores and loads share one completion
  // counter, so stores in the loop delay every later load wait).
  float *score_row[G];
#pragma unroll
  for (int i = 0; i < G; ++i) score_row[i] = scores ? scores + (int64_t)(qh0 + i) * cap : nullptr;

  // KPC: q_c * alpha_c * 2^-cls (qa) and 2^-24 sum_c q_c beta_c (b24) of
  // the lane's channels for key block kblk
  float qa[KPC ? G : 1][KPC ? CPL : 1], b24[KPC ? G : 1];
  int kblk = -1;
  const rsrc_t rkb = KPC ? make_rsrc(A.lo_kb + ((int64_t)h * A.n_kblk) * kHeadDim, (uint32_t)A.n_kblk * kHeadDim * 4u)
                         : r_none;
  auto kpc_refresh = [&](int blk) {
    if constexpr (KPC) {
      uint32_t pw[CPL];
#pragma unroll
      for (int j = 0; j < CPL / 4; ++j) {
        auto w = __builtin_amdgcn_raw_buffer_load_b128(rkb, ((uint32_t)blk * kHeadDim + part * CPL + 4 * j) * 4u, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) pw[4 * j + e] = w[e];
      }
#pragma unroll
      for (int i = 0; i < G; ++i) {
        float bs = 0.0f;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const float sc = __builtin_ldexpf(1.0f, -F::cls(p));
#pragma unroll
          for (int side = 0; side < 2; ++side) {
            const int c = side ? F::hi(p) : F::lo(p);
            const float a = f16_to_f32((uint16_t)(pw[c] & 0xffffu)), b = f16_to_f32((uint16_t)(pw[c] >> 16));
            qa[i][c] = (qkeep[i][c] * a) * sc;
            bs = fmaf(qkeep[i][c], b, bs);
          }
        }
        b24[i] = __builtin_ldexpf(bs, -24);
      }
      kblk = blk;
    }
  };

  float s2[UNROLL][S];
  bool valid[UNROLL];
  // Scores of one iteration (and the lazy running-max update).
  auto proc_k = [&](Rows<BITS, CPL>(&cur)[UNROLL], int it) {
    uint64_t raise = 0;  // lanes whose score passes the lazy threshold (a ballot per token)
    if constexpr (RULES) it = it_end - 1 - it;
    const int rem = end - it * kPerIter;  // wave-uniform: a token is valid when first + u * TPW < rem
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      valid[u] = first < rem - u * TPW;
      if constexpr (RULES) valid[u] = valid[u] && (int)cur[u].pos >= begin;
      uint32_t kx[NP], kraw[Rows<BITS, CPL>::KW];
      seg_words(cur[u].k, kraw);
      FK::template unpack<CPL>(kraw, kx);
      const half2_t kab = as_h2(cur[u].kp);  // (alpha, beta) of the key group
      if constexpr (KPC) {
        // the token's key block (the parameter word is its position); tokens
        // past the pool read position 0 and are masked below
        const int blk = min(max((int)cur[u].kp / kKeyBlock, 0), max(A.n_kblk - 1, 0));
        if (blk != kblk) kpc_refresh(blk);
      }
      float sums[G];
#pragma unroll
      for (int i = 0; i < G; ++i) {
        float d = 0.0f;
        if constexpr (KPC) {
          // 2^-24 sum_c q_c alpha_c code_c: each masked code is an exact
          // fp16 subnormal (code * 2^(cls - 24)) in a mixed-precision FMA
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            const half2_t hk = as_h2(kx[p]);
            d = fmaf(qa[i][F::lo(p)], (float)hk.x, d);
            d = fmaf(qa[i][F::hi(p)], (float)hk.y, d);
          }
        } else {
#pragma unroll
          for (int p = 0; p < NP; ++p) d = __builtin_amdgcn_fdot2(as_h2(kx[p]), qh[i][p], d, false);
          if constexpr (SPLITQ) {
#pragma unroll
            for (int p = 0; p < NP; ++p) d = __builtin_amdgcn_fdot2(as_h2(kx[p]), ql[i][p], d, false);
          }
        }
        // 2^-24 (alpha * 2^24 * d + beta * qsum): the fp16 scale and zero
        // enter mixed-precision FMAs as stored; the power of two goes into
        // the final scale, so the result is the same bits
        float s = KPC ? d + b24[i] : Q ? fmaf((float)kab.x, d, fmaf((float)kab.y, qsum24[i], 0.0f)) : d;
        if constexpr (RULES) {
          sums[i] = s;
          continue;
        }
        s = token_sum<LPT>(s) * s2scale_q;
        s = valid[u] ? s : kNegInf;
        s2[u][i % S] = s;
        // every lane of the token holds s: all of them store it (same
        // value, same address), which keeps the loop free of exec-mask
        // branches around the store
        s_lds[i * max_chunk(G) + it * kPerIter + u * TPW + tsub] = s;
        raise |= __ballot(s > m2[i % S] + kLazy);
      }
      if constexpr (RULES) {
        const float dot = token_sum_own<LPT, G>(sums);
        float s = rule_score(A.rules, dot * s2scale_q, dot * arg_scale, slope2, (int)cur[u].pos);
        s = valid[u] ? s : kNegInf;
        s2[u][0] = s;
        s_lds[own * max_chunk(G) + it * kPerIter + u * TPW + tsub] = s;
        raise |= __ballot(s > m2[0] + kLazy);
      }
    }
    if constexpr (RULES) {
      if (raise) {
        float mx = s2[0][0], f[G];
#pragma unroll
        for (int u = 1; u < UNROLL; ++u) mx = fmaxf(mx, s2[u][0]);
        mx = fmaxf(over_lanes<G>(mx, [](float x, float y) { return fmaxf(x, y); }), m2[0]);
        const float fo = m2[0] == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(m2[0] - mx);
        m2[0] = mx;
        l[0] *= fo;
        token_share<G>(fo, f);
#pragma unroll
        for (int i = 0; i < G; ++i) {
          bsum[i] *= f[i];
#pragma unroll
          for (int c = 0; c < CPL; ++c) o[i][c] *= f[i];
        }
      }
    } else if (raise) {
#pragma unroll
      for (int i = 0; i < S; ++i) {
        float mx = s2[0][i];
#pragma unroll
        for (int u = 1; u < UNROLL; ++u) mx = fmaxf(mx, s2[u][i]);
        mx = wave_max(mx);
        if (mx > m2[i]) {
          const float f = m2[i] == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(m2[i] - mx);
          l[i] *= f;
          bsum[i] *= f;
#pragma unroll
          for (int c = 0; c < CPL; ++c) o[i][c] *= f;
          m2[i] = mx;
        }
      }
    }
  };
  // Value sums of one iteration.
  auto proc_v = [&](Rows<BITS, CPL>(&cur)[UNROLL]) {
    // RULES: until a visible token raises it the maximum stays at -inf, where
    // every score is, too
    const float ref = RULES && m2[0] == kNegInf ? 0.0f : m2[0];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const bool hidden = RULES && !valid[u];
      uint32_t vx[NP], vraw[Rows<BITS, CPL>::KW];
      seg_words(cur[u].v, vraw);
      F::template unpack<CPL>(vraw, vx);
      if constexpr (RULES && !Q) {
#pragma unroll
        for (int p = 0; p < NP; ++p) vx[p] = hidden ? 0u : vx[p];
      }
      const half2_t vab = as_h2(hidden ? 0u : cur[u].vp);  // (alpha, beta) of the value group
      float shared[G];
      if constexpr (RULES) {
        const float e = __builtin_amdgcn_exp2f(s2[u][0] - ref);
        l[0] += e;
        token_share<G>(e, shared);
      }
#pragma unroll
      for (int i = 0; i < G; ++i) {
        // past the pool s2 = -inf, and m2 is finite from the first iteration
        // on (its first token is valid and raises the max), so e = 0
        const float e = RULES ? shared[i] : __builtin_amdgcn_exp2f(s2[u][i % S] - m2[i % S]);
        if constexpr (!RULES) l[i % S] += e;
        const float w = Q ? fmaf(e, (float)vab.x, 0.0f) : e;
        if constexpr (Q) bsum[i] = fmaf(e, (float)vab.y, bsum[i]);
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const half2_t hv = as_h2(vx[p]);
          o[i][F::lo(p)] = fmaf(w, (float)hv.x, o[i][F::lo(p)]);
          o[i][F::hi(p)] = fmaf(w, (float)hv.y, o[i][F::hi(p)]);
        }
      }
    }
  };
  auto proc = [&](Rows<BITS, CPL>(&cur)[UNROLL], int it) {
    proc_k(cur, it);
    proc_v(cur);
  };

  // Software pipeline: the rows of the next PREFETCH iterations are loaded
  // while the current one is computed.  PREFETCH < 0: half steps in the
  // same registers -- the next iteration's keys are loaded as soon as the
  // scores are done, its values as soon as the value sums are, so one half
  // of the rows is always in flight without extra registers.
  if constexpr (PREFETCH < 0) {
    // (no branch around the loads, and scheduling barriers: a load issued
    // early would need registers of its own)
    for (int it = 0; it < n_iter; ++it) {
      const bool live = it + 1 < n_iter;
      proc_k(cur, it);
      __builtin_amdgcn_sched_barrier(0);
      load_part(std::integral_constant<int, 1>{}, cur, it + 1, live);
      __builtin_amdgcn_sched_barrier(0);
      proc_v(cur);
      __builtin_amdgcn_sched_barrier(0);
      load_part(std::integral_constant<int, 2>{}, cur, it + 1, live);
      __builtin_amdgcn_sched_barrier(0);
    }
  } else if constexpr (PREFETCH == 0) {
    for (int it = 0; it < n_iter; ++it) {
      if (it > 0) load_it(cur, it);
      proc(cur, it);
    }
  } else if constexpr (PREFETCH == 1) {
    for (int it = 0; it < n_iter; ++it) {
      proc(cur, it);
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) cur[u] = n1[u];
      if (it + 2 < n_iter) load_it(n1, it + 2);
    }
  } else {
    for (int it = 0; it < n_iter; ++it) {
      proc(cur, it);
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        cur[u] = n1[u];
        n1[u] = n2[u];
      }
      if (it + 3 < n_iter) load_it(n2, it + 3);
    }
  }
  if (scores) {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int i = 0; i < G; ++i)
      for (int j = lane; j < end - start; j += 64)
        __builtin_nontemporal_store(s_lds[i * max_chunk(G) + j], &score_row[i][start + j]);
  }

  // Undo the code scaling, add the beta part, merge the lanes of equal
  // `part` (same channels), and write this chunk's record.
#pragma unroll
  for (int i = 0; i < G; ++i) {
    if constexpr (Q) {
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const float sc = __builtin_ldexpf(1.0f, 24 - F::cls(p));
        o[i][F::lo(p)] = fmaf(o[i][F::lo(p)], sc, bsum[i]);
        o[i][F::hi(p)] = fmaf(o[i][F::hi(p)], sc, bsum[i]);
      }
    }
    if constexpr (!RULES) l[i % S] = wave_sum(l[i % S]) * (1.0f / LPT);  // every lane of a token added its e
#pragma unroll
    for (int c = 0; c < CPL; ++c) o[i][c] = sum_token_lanes<LPT>(o[i][c]);
  }
  if constexpr (RULES) {  // over the lanes of this lane's head, LPT / G of them per token
    l[0] = over_lanes<G>(l[0], [](float x, float y) { return x + y; }) * ((float)G / LPT);
  }
  const int nc = A.nc_hi + A.nc_lo;
#pragma unroll
  for (int i = 0; i < G; ++i) {
    float *rec = A.partials + ((int64_t)(qh0 + i) * nc + rec_chunk) * kRec;
    if (lane == (RULES ? i : 0)) {
      rec[0] = m2[i % S];
      rec[1] = l[i % S];
      rec[kRecN] = __builtin_bit_cast(float, n_pool);
    }
    if (tsub == 0) {
#pragma unroll
      for (int c = 0; c < CPL / 4; ++c)
        *reinterpret_cast<float4 *>(rec + kRecO + chan8(c >> 1) + 4 * (c & 1)) =
            make_float4(o[i][4 * c], o[i][4 * c + 1], o[i][4 * c + 2], o[i][4 * c + 3]);
    }
  }
}

// ---------------------------------------------------------------------------
// The 2-bit retained pool on the matrix cores (16x16x32 fp16 MFMA).
//
// Lane l = 16 a + n.  Scores of a 16-token tile: B holds the tile's key
// codes as exact fp16 subnormals: the 2-bit field of class k (its position
// in the byte) is shifted to mantissa bits 6-7 (k even: code * 2^-18) or
// 8-9 (k odd: code * 2^-16) of its 16-bit half.  The matrix cores multiply
// the deepest fp16 subnormals (code * 2^-24, 2^-22) at reduced precision,
// about 5e-6 relative, but subnormals from 2^-18 up exactly (measured).
// Lane (n, a) holds the 32 codes of channels [32a, 32a + 32) of token n, so
// the token-major key rows are read as they are stored.  A
// holds the query: row 4 s + gamma carries q_hat (times 2^qshift, and 4 more
// for even classes, so every product is q * code * 2^(qshift - 16)) of query
// slot s on the channels of quantization group gamma and 0 elsewhere, so
// lane (n, a) receives, for query slot a, one partial dot product per group
// and applies token n's per-group scale and zero (folded Eq. 1).
//
// Value sums: the pool's value codes are stored in 32-slot tiles
// (int2_v_byte): lane (n, g) reads, in one 16-byte load, bytes n and n + 16
// of slots 8g..8g+7, whose fields are channels n + 32j and n + 16 + 32j.
// For n-block nb (channels 16nb..16nb+15) it takes field nb/2 of byte
// n + 16(nb%2), moved to bits 8-9 of its half: B = codes * 2^-16 (tokens x
// channels, the scale undone on the output); A = the softmax weights
// e * alpha of the column's group,
// split in an fp16 high and low part (rows 2i and 2i+1 for query i) and
// staged through LDS into the operand layout.
// ---------------------------------------------------------------------------
typedef _Float16 h8_t __attribute__((ext_vector_type(8)));
typedef float f4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u4_t __attribute__((ext_vector_type(4)));

__device__ inline h8_t pack_h8(uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  const u4_t u = {x, y, z, w};
  return __builtin_bit_cast(h8_t, u);
}

__device__ inline f4_t mfma32(h8_t a, h8_t b, f4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Reductions over the 16 lanes of each row (lane group); result in all 16.
__device__ inline float row_max16(float v) {
  v = fmaxf(v, dpp_mov<0xB1>(v));
  v = fmaxf(v, dpp_mov<0x4E>(v));
  v = fmaxf(v, dpp_mov<0x141>(v));
  return fmaxf(v, dpp_mov<0x140>(v));
}
__device__ inline float row_sum16(float v) {
  v += dpp_mov<0xB1>(v);
  v += dpp_mov<0x4E>(v);
  v += dpp_mov<0x141>(v);
  return v + dpp_mov<0x140>(v);
}

#ifndef MIKV_INT2_KEY_TILES
#define MIKV_INT2_KEY_TILES 2
#endif
constexpr int kKT = MIKV_INT2_KEY_TILES;  // 16-token key tiles per iteration (2 or 4)
constexpr int kVT = kKT / 2;              // 32-token value tiles per iteration
constexpr int kItTok = 16 * kKT;          // tokens per iteration
// Operand element -> slot inside a lane group's 8 (and back): bits 0 and 1
// swapped, the order the masked code pairs come out in.
__host__ __device__ constexpr int tau8(int e) { return (e & 4) | ((e & 1) << 1) | ((e >> 1) & 1); }

// LDS weight staging: [group][value tile][row 0..15][lane group][element]
// halves; rows past 2G stay zero, so every lane reads its operand.
__device__ inline int w_index(int gamma, int vt, int row, int g, int e) {
  return (((gamma * kVT + vt) * 16 + row) * 4 + g) * 8 + e;
}
constexpr int kWLds = 4 * kVT * 16 * 4 * 8;  // halves (4 KiB per value tile)

template <int G, bool SPLITQ, int NG, bool STREAM, bool RULES = false>
__device__ void attn_chunk_int2(const AttnArgs &A, int h, int chunk, int rec_chunk, float *s_lds, _Float16 *w_lds) {
  constexpr int QS = G < 4 ? G : 4;    // distinct query slots in one row block
  constexpr int NSET = G > 4 ? 2 : 1;  // query sets (G = 8: queries 0-3 and 4-7)
  constexpr int R = 4 / QS;            // lane groups holding the same query slot
  constexpr int NGL = (NG + R - 1) / R;  // value groups each lane weights
  constexpr int NP = SPLITQ ? 2 : 1;   // fp16 parts of the query
  constexpr int GROUP = kHeadDim / NG;
  constexpr int kCpol = STREAM ? kStreamPolicy : 0;
  const int lane = threadIdx.x & 63, n = lane & 15, a = lane >> 4;
  const int qs = a % QS, rho = a / QS;
  const int b = h / A.kv_heads, kvh = h % A.kv_heads;
  const int qh0 = b * A.q_heads + kvh * G;
  const int cap = A.cap_lo;
  const int n_pool = __builtin_amdgcn_readfirstlane(A.n_lo[h]);
  const int start = chunk * A.chunk_lo;
  const int end = min(start + A.chunk_lo, n_pool);
  int n_iter = end > start ? (end - start + kItTok - 1) / kItTok : 0;
  float *scores = A.scores_lo;

  const rsrc_t rk = make_rsrc(A.lo_k + (int64_t)h * cap * 32, (uint32_t)n_pool * 32u);
  const rsrc_t rv = make_rsrc(A.lo_v + (int64_t)h * cap * 32, (uint32_t)((n_pool + 31) / 32) * 1024u);
  const rsrc_t rkp = make_rsrc(A.lo_kp + (int64_t)h * cap * NG, (uint32_t)n_pool * NG * 4u);
  const rsrc_t rvp = make_rsrc(A.lo_vp + (int64_t)h * cap * NG, (uint32_t)n_pool * NG * 4u);
  const rsrc_t rpos = make_rsrc(RULES ? (const void *)(A.lo_pos + (int64_t)h * cap) : (const void *)A.lo_k,
                                RULES && rule_positions(A.rules) ? (uint32_t)n_pool * 4u : 0u);

  int begin = 0, it_end = n_iter;
  if constexpr (RULES) {
    begin = rule_begin(A.rules, b);
    int it_begin = 0;
    visible_range<kItTok>(A.rules, rpos, begin, start, end, it_begin, it_end);
    if (it_end - it_begin < n_iter && scores) {
      for (int i = 0; i < G; ++i)
        for (int j = lane; j < end - start; j += 64) s_lds[i * max_chunk(G) + j] = kNegInf;
    }
    n_iter = it_end - it_begin;
  }

  // One iteration's loads: key codes and parameter rows of the four key
  // tiles (the lane's value groups only), value codes of the two tiles.
  struct Ld {
    uint32_t kc[kKT][2];
    uint32_t kp[kKT][NG];
    uint32_t vp[kKT][NGL];
    uint32_t vc[kVT][4];
    uint32_t pos[RULES ? kKT : 1];
  };
  // KEYS: the key codes and parameters; VALS: the value codes and
  // parameters.  With `live` false every load goes through an empty
  // descriptor (zero, no memory access), so no branch is needed around it.
  const rsrc_t r_none = make_rsrc(A.lo_k, 0u);
  auto load = [&](Ld &d, int it, bool keys, bool vals, bool live) {
    const uint32_t t0 = (uint32_t)(start + (RULES ? it_end - 1 - it : it) * kItTok);
    const rsrc_t ak = live ? rk : r_none, av = live ? rv : r_none;
    const rsrc_t akp = live ? rkp : r_none, avp = live ? rvp : r_none;
#pragma unroll
    for (int q = 0; q < kKT; ++q) {
      const uint32_t slot = t0 + 16 * q + n;
      if (RULES && keys) d.pos[q] = __builtin_amdgcn_raw_buffer_load_b32(live ? rpos : r_none, slot * 4u, 0, kCpol);
      if (keys) {
        auto kc = __builtin_amdgcn_raw_buffer_load_b64(ak, slot * 32u + 8u * a, 0, kCpol);
        d.kc[q][0] = kc[0];
        d.kc[q][1] = kc[1];
        if constexpr (NG == 4) {
          auto kp = __builtin_amdgcn_raw_buffer_load_b128(akp, slot * 16u, 0, kCpol);
#pragma unroll
          for (int j = 0; j < 4; ++j) d.kp[q][j] = kp[j];
        } else if constexpr (NG == 2) {
          auto kp = __builtin_amdgcn_raw_buffer_load_b64(akp, slot * 8u, 0, kCpol);
          d.kp[q][0] = kp[0];
          d.kp[q][1] = kp[1];
        } else {
          d.kp[q][0] = __builtin_amdgcn_raw_buffer_load_b32(akp, slot * 4u, 0, kCpol);
        }
      }
      if (vals) {
        if constexpr (R == 1 && NG == 4) {  // every group: the whole row, one load
          auto vp = __builtin_amdgcn_raw_buffer_load_b128(avp, slot * 16u, 0, kCpol);
#pragma unroll
          for (int j = 0; j < 4; ++j) d.vp[q][j] = vp[j];
        } else if constexpr (R == 1 && NG == 2) {
          auto vp = __builtin_amdgcn_raw_buffer_load_b64(avp, slot * 8u, 0, kCpol);
          d.vp[q][0] = vp[0];
          d.vp[q][1] = vp[1];
        } else {
#pragma unroll
          for (int j = 0; j < NGL; ++j)
            d.vp[q][j] = __builtin_amdgcn_raw_buffer_load_b32(avp, (slot * NG + (uint32_t)((rho + R * j) % NG)) * 4u, 0, kCpol);
        }
      }
    }
    if (vals) {
#pragma unroll
      for (int vt = 0; vt < kVT; ++vt) {
        const uint32_t tile = (t0 >> 5) + vt;
        auto vc = __builtin_amdgcn_raw_buffer_load_b128(av, tile * 1024u + 16u * (uint32_t)lane, 0, kCpol);
#pragma unroll
        for (int j = 0; j < 4; ++j) d.vc[vt][j] = vc[j];
      }
    }
  };
  Ld cur;
  load(cur, 0, true, true, n_iter > 0);

  // zero the weight rows (rows past 2G are never written)
  {
    uint4 *w4 = reinterpret_cast<uint4 *>(w_lds);
#pragma unroll
    for (int j = 0; j < kWLds / 8 / 64; ++j) w4[j * 64 + lane] = make_uint4(0u, 0u, 0u, 0u);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }

  // Query operands.  As an A row, lane l is row m = n: query slot m/4 (mod
  // QS) of set st, group m%4, over K block a (channels [32a, 32a + 32)).
  h8_t AK[NSET][NP][4];
  float qpart[NSET];
  // the query scaled by 2^(qshift - 2 k) for class k (query_shift)
  float qfs[NSET][32];
  float qmax = 0.0f;
#pragma unroll
  for (int st = 0; st < NSET; ++st) {
    const int iq = (n / 4) % QS + 4 * st;
    const uint4 *q4 = reinterpret_cast<const uint4 *>(A.q + (int64_t)(qh0 + iq) * kHeadDim + 32 * a);
    uint4 qr[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) qr[j] = q4[j];
    float *qf = qfs[st];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t w[4] = {qr[j].x, qr[j].y, qr[j].z, qr[j].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        qf[8 * j + 2 * k] = f16_to_f32((uint16_t)(w[k] & 0xffffu));
        qf[8 * j + 2 * k + 1] = f16_to_f32((uint16_t)(w[k] >> 16));
      }
    }
    if constexpr (SPLITQ) {
      const float4 *b4 = reinterpret_cast<const float4 *>(A.balance + (int64_t)h * kHeadDim + 32 * a);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float4 v = b4[j];
        qf[4 * j] = qf[4 * j] / v.x;
        qf[4 * j + 1] = qf[4 * j + 1] / v.y;
        qf[4 * j + 2] = qf[4 * j + 2] / v.z;
        qf[4 * j + 3] = qf[4 * j + 3] / v.w;
      }
    }
#pragma unroll
    for (int j = 0; j < 32; ++j) qmax = fmaxf(qmax, fabsf(qf[j]));
  }
  // the even-class query operand carries 2^(qshift + 2): largest qshift in
  // {6, 4, 2, 0} that keeps it within fp16 (wave-uniform)
  const float qm = wave_max(qmax);
  const int qshift = qm * 256.0f < 60000.0f ? 6 : qm * 64.0f < 60000.0f ? 4 : qm * 16.0f < 60000.0f ? 2 : 0;
  const float s2scale_q = __builtin_ldexpf(A.scale * kLog2e, 16 - qshift);
  float arg_scale = 0.0f, slope2[RULES ? NSET : 1];  // slopes of the lane's own queries
  if constexpr (RULES) {
    arg_scale = __builtin_ldexpf(A.rules.cap_scale, 16 - qshift);
#pragma unroll
    for (int st = 0; st < NSET; ++st) slope2[st] = A.rules.slopes ? A.rules.slopes[kvh * G + qs + 4 * st] * kLog2e : 0.0f;
  }
#pragma unroll
  for (int st = 0; st < NSET; ++st) {
    const float *qf = qfs[st];
    float ps = 0.0f;
#pragma unroll
    for (int j = 0; j < 32; ++j) ps += qf[j];
    qpart[st] = ps;
    const float keep = (32 * a) / GROUP == n % 4 ? 1.0f : 0.0f;  // the lane's channels lie in one group
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t hw[4], lw[4];
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        float vv[2];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const int e = 2 * d + hf;
          const int j = 16 * (i >> 1) + 4 * (i & 1) + (e >> 1) + 8 * (e & 1);
          vv[hf] = qf[j] * (keep * __builtin_ldexpf(1.0f, qshift + ((e >> 1) & 1 ? 0 : 2)));
        }
        const _Float16 h0 = (_Float16)vv[0], h1 = (_Float16)vv[1];
        hw[d] = (uint32_t)__builtin_bit_cast(uint16_t, h0) | ((uint32_t)__builtin_bit_cast(uint16_t, h1) << 16);
        if constexpr (SPLITQ) {
          const _Float16 l0 = (_Float16)(vv[0] - (float)h0), l1 = (_Float16)(vv[1] - (float)h1);
          lw[d] = (uint32_t)__builtin_bit_cast(uint16_t, l0) | ((uint32_t)__builtin_bit_cast(uint16_t, l1) << 16);
        }
      }
      AK[st][0][i] = pack_h8(hw[0], hw[1], hw[2], hw[3]);
      if constexpr (SPLITQ) AK[st][NP - 1][i] = pack_h8(lw[0], lw[1], lw[2], lw[3]);
    }
  }
  // Sum of q_hat over each group for the lane's own query slot (the zero
  // term of the folded dequantization), from the rows 4 s of lane groups a'.
  float qsl[NSET][NG];
#pragma unroll
  for (int st = 0; st < NSET; ++st) {
    float all[QS][NG];
#pragma unroll
    for (int s3 = 0; s3 < QS; ++s3) {
#pragma unroll
      for (int gm = 0; gm < NG; ++gm) all[s3][gm] = 0.0f;
#pragma unroll
      for (int ap = 0; ap < 4; ++ap) all[s3][(32 * ap) / GROUP] += lane_value(qpart[st], 16 * ap + 4 * s3);
    }
#pragma unroll
    for (int gm = 0; gm < NG; ++gm) {
      float v = all[0][gm];
#pragma unroll
      for (int s3 = 1; s3 < QS; ++s3) v = qs == s3 ? all[s3][gm] : v;
      qsl[st][gm] = __builtin_ldexpf(v, qshift - 16);  // 2^(qshift - 16): the scale of the scores below
    }
  }

  float m2q[G];       // running max per query (wave-uniform, log2 units)
  float m_own[NSET];  // the max of the lane's own query
#pragma unroll
  for (int i = 0; i < G; ++i) m2q[i] = kNegInf;
#pragma unroll
  for (int st = 0; st < NSET; ++st) m_own[st] = kNegInf;
  float l_l[NSET], bs_l[NSET][NGL];
#pragma unroll
  for (int st = 0; st < NSET; ++st) {
    l_l[st] = 0.0f;
#pragma unroll
    for (int j = 0; j < NGL; ++j) bs_l[st][j] = 0.0f;
  }
  // a lane's duplicate value group (fewer groups than replicas) adds nothing
  float dup[NGL];
#pragma unroll
  for (int j = 0; j < NGL; ++j) dup[j] = rho + R * j < NG ? 1.0f : 0.0f;
  f4_t CV[8];
#pragma unroll
  for (int nb = 0; nb < 8; ++nb) CV[nb] = f4_t{0.0f, 0.0f, 0.0f, 0.0f};
  // value fields go to bits 8-9 of each half (code * 2^-16)
  constexpr uint32_t mk = 0x03000300u;

  // Half-step pipeline (as in attn_chunk): the next iteration's keys are
  // loaded once the scores are done, its values once the value MFMAs are.
  for (int it = 0; it < n_iter; ++it) {
    const bool live = it + 1 < n_iter;
    const int t0 = start + (RULES ? it_end - 1 - it : it) * kItTok;
    // --- scores of the four key tiles
    float s2[kKT][NSET];
    uint64_t raise = 0;
#pragma unroll
    for (int q = 0; q < kKT; ++q) {
      // code pairs of bytes 0, 2 (fields k at bits 2k) and bytes 1, 3
      // (bits 8 + 2k), each field moved to bits 6-7 (k even) or 8-9 (k odd)
      // of its half: code * 2^-18 or code * 2^-16
      uint32_t P[16];
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const uint32_t x = cur.kc[q][w];
        const uint32_t l6 = x << 6, l2 = x << 2, r2 = x >> 2, r6 = x >> 6;
        P[(2 * w) * 4 + 0] = l6 & 0x00c000c0u;
        P[(2 * w) * 4 + 1] = l6 & 0x03000300u;
        P[(2 * w) * 4 + 2] = l2 & 0x00c000c0u;
        P[(2 * w) * 4 + 3] = l2 & 0x03000300u;
        P[(2 * w + 1) * 4 + 0] = r2 & 0x00c000c0u;
        P[(2 * w + 1) * 4 + 1] = r2 & 0x03000300u;
        P[(2 * w + 1) * 4 + 2] = r6 & 0x00c000c0u;
        P[(2 * w + 1) * 4 + 3] = r6 & 0x03000300u;
      }
      bool valid = t0 + 16 * q + n < end;
      if constexpr (RULES) valid = valid && (int)cur.pos[q] >= begin;
#pragma unroll
      for (int st = 0; st < NSET; ++st) {
        f4_t C = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int pt = 0; pt < NP; ++pt)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            C = mfma32(AK[st][pt][i], pack_h8(P[4 * i], P[4 * i + 1], P[4 * i + 2], P[4 * i + 3]), C);
        // 2^(qshift - 16) times the folded score (the fp16 scale and zero enter
        // mixed-precision FMAs as stored; the power of two is in the scale)
        // (two independent chains: no dependent mixed FMAs back to back)
        float sp[2] = {0.0f, 0.0f};
#pragma unroll
        for (int gm = 0; gm < NG; ++gm) {
          const half2_t kab = as_h2(cur.kp[q][gm]);
          sp[gm & 1] = fmaf((float)kab.x, C[gm], fmaf((float)kab.y, qsl[st][gm], sp[gm & 1]));
        }
        // -inf for a token past the chunk, as a select (no branch)
        float v2;
        if constexpr (RULES) {
          const float dot = sp[0] + sp[1];
          v2 = rule_score(A.rules, dot * s2scale_q, dot * arg_scale, slope2[st], (int)cur.pos[q]);
          v2 = valid ? v2 : kNegInf;
        } else {
          v2 = fmaf(sp[0] + sp[1], s2scale_q, valid ? 0.0f : kNegInf);
        }
        s2[q][st] = v2;
        if (scores) s_lds[(qs + 4 * st) * max_chunk(G) + (t0 - start) + 16 * q + n] = v2;  // replicas agree
        raise |= __ballot(v2 > m_own[st] + kLazy);
      }
    }
    // --- lazy running max (per query; rare after the first tokens)
    if (raise) {
      float f[G];
#pragma unroll
      for (int i = 0; i < G; ++i) f[i] = 1.0f;
#pragma unroll
      for (int st = 0; st < NSET; ++st) {
        float mx = s2[0][st];
#pragma unroll
        for (int q = 1; q < kKT; ++q) mx = fmaxf(mx, s2[q][st]);
        mx = row_max16(mx);
        float ra[4];
#pragma unroll
        for (int ap = 0; ap < 4; ++ap) ra[ap] = lane_value(mx, 16 * ap);
#pragma unroll
        for (int s3 = 0; s3 < QS; ++s3) {
          float qm = kNegInf;
#pragma unroll
          for (int ap = 0; ap < 4; ++ap)
            if (ap % QS == s3) qm = fmaxf(qm, ra[ap]);
          const int iq = s3 + 4 * st;
          if (qm > m2q[iq]) {
            f[iq] = m2q[iq] == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(m2q[iq] - qm);
            m2q[iq] = qm;
          }
        }
      }
#pragma unroll
      for (int st = 0; st < NSET; ++st) {
        float fo = f[4 * st], mo = m2q[4 * st];
#pragma unroll
        for (int s3 = 1; s3 < QS; ++s3) {
          fo = qs == s3 ? f[s3 + 4 * st] : fo;
          mo = qs == s3 ? m2q[s3 + 4 * st] : mo;
        }
        m_own[st] = mo;
        l_l[st] *= fo;
#pragma unroll
        for (int j = 0; j < NGL; ++j) bs_l[st][j] *= fo;
      }
      // value accumulators: register r of lane group a is row 4a + r, query (4a + r) / 2
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float fr = 1.0f;
#pragma unroll
        for (int i = 0; i < G; ++i) fr = (4 * a + r) / 2 == i ? f[i] : fr;
#pragma unroll
        for (int nb = 0; nb < 8; ++nb) CV[nb][r] *= fr;
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    load(cur, it + 1, true, false, live);
    __builtin_amdgcn_sched_barrier(0);
    // --- weights e * alpha into LDS (the A layout of the value MFMAs)
#pragma unroll
    for (int q = 0; q < kKT; ++q) {
      const int p = 16 * q + n, vt = p >> 5, u = p & 31;
      const int gv = u >> 3, ei = tau8(u & 7);
#pragma unroll
      for (int st = 0; st < NSET; ++st) {
        const int iq = qs + 4 * st;
        // (RULES: the maximum is -inf until a visible token raises it; a hidden
        // token's parameters count as 0, whatever they are)
        const bool hidden = RULES && s2[q][st] == kNegInf;
        const float e = __builtin_amdgcn_exp2f(s2[q][st] - (RULES && m_own[st] == kNegInf ? 0.0f : m_own[st]));  // 0 for -inf scores
        l_l[st] += e;
#pragma unroll
        for (int j = 0; j < NGL; ++j) {
          const int gm = (rho + R * j) % NG;
          const half2_t vab = as_h2(hidden ? 0u : cur.vp[q][j]);  // (alpha, beta) of the value group
          bs_l[st][j] = fmaf(e * dup[j], (float)vab.y, bs_l[st][j]);
          // e * alpha as fp16 high and low parts, each one mixed FMA: the low
          // part rounds the exact residual e * alpha - high
          const _Float16 wh = (_Float16)fmaf(e, (float)vab.x, 0.0f);
          const _Float16 wl = (_Float16)fmaf(e, (float)vab.x, -(float)wh);
          w_lds[w_index(gm, vt, 2 * iq, gv, ei)] = wh;
          w_lds[w_index(gm, vt, 2 * iq + 1, gv, ei)] = wl;
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    // --- value MFMAs
#pragma unroll
    for (int vt = 0; vt < kVT; ++vt) {
      h8_t AV[NG];
#pragma unroll
      for (int gm = 0; gm < NG; ++gm) AV[gm] = *reinterpret_cast<const h8_t *>(w_lds + w_index(gm, vt, n, a, 0));
#pragma unroll
      for (int nb = 0; nb < 8; ++nb) {
        // channels 16 nb + n: segment j = nb / 2 (field j of every byte),
        // bytes n + 16 (nb % 2) of the lane's 8 slots
        const int j = nb >> 1;
        const uint32_t d0 = cur.vc[vt][2 * (nb & 1)], d1 = cur.vc[vt][2 * (nb & 1) + 1];
        CV[nb] = mfma32(AV[(16 * nb) / GROUP],
                        pack_h8((d0 << (8 - 2 * j)) & mk, (d0 >> (2 * j)) & mk, (d1 << (8 - 2 * j)) & mk,
                                (d1 >> (2 * j)) & mk),
                        CV[nb]);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    load(cur, it + 1, false, true, live);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }

  // Scores of the chunk: one burst from LDS.
  const int nc = A.nc_hi + A.nc_lo;
  if (scores) {
#pragma unroll
    for (int i = 0; i < G; ++i) {
      float *row = scores + (int64_t)(qh0 + i) * cap;
      for (int j = lane; j < end - start; j += 64) __builtin_nontemporal_store(s_lds[i * max_chunk(G) + j], &row[start + j]);
    }
  }
  // Normalisers and zero terms per (query, group), wave-uniform.
  float lq[G], bq[G][NG];
#pragma unroll
  for (int st = 0; st < NSET; ++st) {
    const float lr = row_sum16(l_l[st]);
    float br[NGL];
#pragma unroll
    for (int j = 0; j < NGL; ++j) br[j] = row_sum16(bs_l[st][j]);
#pragma unroll
    for (int s3 = 0; s3 < QS; ++s3) {
      const int iq = s3 + 4 * st;
      lq[iq] = lane_value(lr, 16 * s3);  // replica 0 of the slot
#pragma unroll
      for (int gm = 0; gm < NG; ++gm) bq[iq][gm] = lane_value(br[gm / R], 16 * (s3 + QS * (gm % R)));
    }
  }
  // Record per query: max, normaliser, value sums (lane group i/2 holds
  // query i in registers 2(i%2), 2(i%2)+1).
  constexpr float colscale = 65536.0f;  // undoes the value encoding (code * 2^-16)
#pragma unroll
  for (int i = 0; i < G; ++i) {
    float *rec = A.partials + ((int64_t)(qh0 + i) * nc + rec_chunk) * kRec;
    if (lane == 0) {
      rec[0] = m2q[i];
      rec[1] = lq[i];
      rec[kRecN] = __builtin_bit_cast(float, n_pool);
    }
    if (a == i / 2) {
      const int r0 = 2 * (i % 2);
#pragma unroll
      for (int nb = 0; nb < 8; ++nb) rec[kRecO + 16 * nb + n] = fmaf(CV[nb][r0] + CV[nb][r0 + 1], colscale, bq[i][(16 * nb) / GROUP]);
    }
  }
}

// Tuning: token tiles per lane per iteration and prefetch depth (-1: the
// half-step pipeline of attn_chunk), for low-bit (INT2/INT4) and high-bit
// (fp16/INT8) rows.
#ifndef MIKV_UNROLL_LOWBIT
#define MIKV_UNROLL_LOWBIT 8
#endif
#ifndef MIKV_UNROLL_HIGHBIT
#define MIKV_UNROLL_HIGHBIT 2
#endif
#ifndef MIKV_PREFETCH_LOWBIT
#define MIKV_PREFETCH_LOWBIT -1
#endif
#ifndef MIKV_PREFETCH_HIGHBIT
#define MIKV_PREFETCH_HIGHBIT -1
#endif
// INT4 rows are twice the INT2 ones: half the tiles per iteration keep the
// same bytes in flight and the registers of one more wave per SIMD.
#ifndef MIKV_UNROLL_INT4
#define MIKV_UNROLL_INT4 4
#endif
// A balanced 2-bit pool (the query in two fp16 parts) takes half the tiles:
// with eight it needs 171 registers and two waves per SIMD, with four 136 and
// three (llama2_13b: 266.6-272.1 -> 261.4-264.4 us per launch, step 303.7-307.4
// -> 299.2-299.8 us; long_context, unbalanced, keeps eight: four measured
// even).
#ifndef MIKV_UNROLL_LOWBIT_SPLIT
#define MIKV_UNROLL_LOWBIT_SPLIT 4
#endif
template <int BITS, bool SPLITQ = false>
constexpr int unroll_for() {
  return BITS == 4 || BITS == 3 ? MIKV_UNROLL_INT4
       : BITS <= 4              ? (SPLITQ ? MIKV_UNROLL_LOWBIT_SPLIT : MIKV_UNROLL_LOWBIT)
                                : MIKV_UNROLL_HIGHBIT;
}
// An fp16 importance pool with one query head per KV head (the least work
// per byte) keeps four tiles in flight (long_context 106.5-107.0 -> 105.0-
// 105.5 us per step); under GQA and for INT8 pools four were slower
// (mistral_7b 87.0 -> 92.8, llama2_7b 44.4 -> 46.0).
#ifndef MIKV_UNROLL_F16_MHA
#define MIKV_UNROLL_F16_MHA 4
#endif
template <int HI, int G>
constexpr int unroll_hi() { return HI == 16 && G == 1 ? MIKV_UNROLL_F16_MHA : unroll_for<HI>(); }
// LEAN: an INT4 retained pool with one query head per KV head and no balancer
// takes two tiles instead of four: fewer registers, one wave more per SIMD,
// which rows from the last-level cache want (partial_lean); an INT3 pool is
// 2 % slower with two.
template <int LO, bool SPLITQ, bool LEAN>
constexpr int unroll_lo() { return LEAN ? 2 : unroll_for<LO, SPLITQ>(); }
template <int BITS>
constexpr int prefetch_for() { return BITS <= 4 ? MIKV_PREFETCH_LOWBIT : MIKV_PREFETCH_HIGHBIT; }

// Query heads per KV head from which a lane holds 16 channels instead of 32
// (fewer accumulators per lane at larger GQA groups).
#ifndef MIKV_NARROW_FROM_G
#define MIKV_NARROW_FROM_G 4
#endif
#ifndef MIKV_WAVES_PER_EU
#define MIKV_WAVES_PER_EU 1
#endif
#ifndef MIKV_CHUNK_KB
#define MIKV_CHUNK_KB 96  // under GQA
#endif
#ifndef MIKV_CHUNK_KB_MHA
#define MIKV_CHUNK_KB_MHA 64  // one query head per KV head (measured: 13B shape -2.5 %, long_context even)
#endif
#ifndef MIKV_CHUNK_HI_SCALE
#define MIKV_CHUNK_HI_SCALE 2  // MHA importance-pool chunks hold this many times the bytes
#endif
#ifndef MIKV_CHUNK_HI_SCALE_F16
#define MIKV_CHUNK_HI_SCALE_F16 4  // the same for an fp16 importance pool
#endif

// The decode step's new token: written into importance-pool slot n_hi by
// the wave whose chunk holds that slot, before the wave reads its chunk (no
// other wave reads the slot, and chunks are whole iterations, so no other
// wave's loads reach it).  A full pool sets the status bit instead (wave
// of chunk 0).
template <int HI>
__device__ inline void append_in_chunk(const AttnArgs &A, int h, int chunk) {
  const int n0 = __builtin_amdgcn_readfirstlane(A.n_hi[h]);
  const int lane = threadIdx.x & 63;
  if (n0 >= A.cap_hi) {
    if (chunk == 0 && lane == 0) atomicOr(A.app.status, MIKV_DEVERR_HI_FULL);
    return;
  }
  if (chunk != n0 / A.chunk_hi) return;
  if (lane < 8) append_row<HI>(A.app, h, n0, lane);
  // the lanes that read the slot see the stored row (one wave per block)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
}

template <int HI, int LO, int G, bool SPLITQ, bool KPC = false, bool LEAN = false, bool RULES = false>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(MIKV_WAVES_PER_EU)))
void attn_partial_kernel(AttnArgs A) {
  constexpr int CPL = G >= MIKV_NARROW_FROM_G ? 16 : 32;  // channels per lane
  // 3-, 4- and 8-bit retained pools at eight query heads per KV head: 8
  // channels per lane (a 3-, 4- or 8-byte segment), so the lane's G x CPL
  // value sums fit the registers of two waves per SIMD instead of spilling
  constexpr int CPL_LO = (LO == 3 || LO == 4 || LO == 8) && G >= 8 ? 8 : CPL;
  // fp16 importance pool: 16 channels per lane in two spread pieces, so the
  // lanes of a token read whole 128-byte lines with each load (which
  // non-temporal loads need to fetch a line once, and which read the
  // resident rows faster too: long_context with an evicting cache 38.9 ->
  // 36.2 us per launch); with eight query heads per KV head 8 channels, which
  // halves the value sums a lane holds (G x CPL registers), and so do INT8
  // and INT4 importance pools at eight.  INT8 below eight: streamed rows 16
  // channels per lane (one piece per line), resident rows the wider lanes,
  // which cost fewer cross-lane sums per token.
  constexpr int CPL_HI = G >= 8 ? 8 : HI == 16 ? 16 : CPL;
  constexpr int CPL_HI_S = G >= 8 ? 8 : HI == 16 || HI == 8 ? 16 : CPL;
  // Block -> (head, chunk): first every head's importance-pool chunks and
  // the retained-pool chunks that cannot be empty (nc_first per head; with
  // pool_major all importance-pool chunks, the longest-running waves of an
  // fp16 pool, before any retained-pool chunk), then
  // the retained-pool chunks that may be (a wave that finds its chunk empty
  // costs little at the end of the grid, but holds up the dispatch of the
  // work behind it anywhere else).
  // Every other step runs the order backwards (A.order, set from the
  // cache length): the last-level cache still holds the end of the previous
  // step's stream, which is then read first.
  const int n_heads = gridDim.x / (A.nc_hi + A.nc_lo);
  const int n_first = n_heads * A.nc_first;  // blocks of the first part
  const int bid = A.order == 2 ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x;
  int h, c;
  if (A.pool_major && bid < n_heads * A.nc_hi) {
    h = bid / A.nc_hi;
    c = bid % A.nc_hi;
  } else if (A.pool_major && bid < n_first) {
    const int e = bid - n_heads * A.nc_hi, per = A.nc_first - A.nc_hi;
    h = e / per;
    c = A.nc_hi + e % per;
  } else if (bid < n_first) {
    h = bid / A.nc_first;
    c = bid % A.nc_first;
  } else {
    const int rest = A.nc_hi + A.nc_lo - A.nc_first, e = bid - n_first;
    h = e / rest;
    c = A.nc_first + e % rest;
  }
  if (A.order == 1) h = n_heads - 1 - h;
  __shared__ float s_lds[G * max_chunk(G)];  // the chunk's scores, [G][max_chunk(G)]
  // The rows of the first res_hi / res_lo heads of each pool (as much as the
  // last-level cache keeps from one step to the next) are read with plain
  // loads, which that cache allocates; all other rows are streamed with
  // non-temporal loads, which do not push the resident rows out.
  if (c < A.nc_hi) {
    if (A.hi_pending) append_in_chunk<HI>(A, h, c);
    if (h < A.res_hi)
      attn_chunk<HI, G, CPL_HI, SPLITQ, unroll_hi<HI, G>(), prefetch_for<HI>(), false, false, RULES>(A, h, c, c, true, s_lds);
    else
      attn_chunk<HI, G, CPL_HI_S, SPLITQ, unroll_hi<HI, G>(), prefetch_for<HI>(), false, true, RULES>(A, h, c, c, true, s_lds);
  } else if constexpr (KPC) {
    attn_chunk<LO, G, CPL, SPLITQ, unroll_for<LO>(), prefetch_for<LO>(), true, false, RULES>(A, h, c - A.nc_hi, c, false, s_lds);
  } else if constexpr (LO == 2 && G >= 2) {
    __shared__ __align__(16) _Float16 w_lds[kWLds];  // value-MFMA weights, see w_index
    const bool res = h < A.res_lo;
    if (A.group == 32) {
      if (res) attn_chunk_int2<G, SPLITQ, 4, false, RULES>(A, h, c - A.nc_hi, c, s_lds, w_lds);
      else attn_chunk_int2<G, SPLITQ, 4, true, RULES>(A, h, c - A.nc_hi, c, s_lds, w_lds);
    } else if (A.group == 64) {
      if (res) attn_chunk_int2<G, SPLITQ, 2, false, RULES>(A, h, c - A.nc_hi, c, s_lds, w_lds);
      else attn_chunk_int2<G, SPLITQ, 2, true, RULES>(A, h, c - A.nc_hi, c, s_lds, w_lds);
    } else {
      if (res) attn_chunk_int2<G, SPLITQ, 1, false, RULES>(A, h, c - A.nc_hi, c, s_lds, w_lds);
      else attn_chunk_int2<G, SPLITQ, 1, true, RULES>(A, h, c - A.nc_hi, c, s_lds, w_lds);
    }
  } else {
    if (h < A.res_lo)
      attn_chunk<LO, G, CPL_LO, SPLITQ, unroll_lo<LO, SPLITQ, LEAN>(), prefetch_for<LO>(), false, false, RULES>(A, h, c - A.nc_hi, c, false, s_lds);
    else
      attn_chunk<LO, G, CPL_LO, SPLITQ, unroll_lo<LO, SPLITQ, LEAN>(), prefetch_for<LO>(), false, true, RULES>(A, h, c - A.nc_hi, c, false, s_lds);
  }
}

template <int HI, int LO, bool SPLITQ, bool RULES>
void launch_partial_q(const AttnArgs &A, int G, bool lean, dim3 grid, hipStream_t st) {
  if constexpr (LO == 4 && !SPLITQ) {
    if (G == 1 && lean) {
      hipLaunchKernelGGL((attn_partial_kernel<HI, LO, 1, SPLITQ, false, true, RULES>), grid, dim3(64), 0, st, A);
      return;
    }
  }
  switch (G) {
    case 1: hipLaunchKernelGGL((attn_partial_kernel<HI, LO, 1, SPLITQ, false, false, RULES>), grid, dim3(64), 0, st, A); break;
    case 2: hipLaunchKernelGGL((attn_partial_kernel<HI, LO, 2, SPLITQ, false, false, RULES>), grid, dim3(64), 0, st, A); break;
    case 4: hipLaunchKernelGGL((attn_partial_kernel<HI, LO, 4, SPLITQ, false, false, RULES>), grid, dim3(64), 0, st, A); break;
    default: hipLaunchKernelGGL((attn_partial_kernel<HI, LO, 8, SPLITQ, false, false, RULES>), grid, dim3(64), 0, st, A); break;
  }
}

// A balanced query (q / b) is not an fp16 value in general: carry it as two
// fp16 parts.  An unbalanced query is fp16 already.
template <int HI, int LO, bool RULES>
void launch_partial_g(const AttnArgs &A, int G, bool lean, dim3 grid, hipStream_t st) {
  if (A.balance)
    launch_partial_q<HI, LO, true, RULES>(A, G, lean, grid, st);
  else
    launch_partial_q<HI, LO, false, RULES>(A, G, lean, grid, st);
}

// The partial phase of cache c (validated; per-channel keys without a balancer).
template <bool RULES>
void launch_partial_c(const AttnArgs &A, const mikv_cache *c, bool lean, dim3 grid, hipStream_t st) {
  const int G = group_size_of(c);
  if (c->key_block) {
    // per-channel retained keys: fp16 importance pool, one query head per KV head, no balancer
    switch (c->lo_bits) {
      case 2: hipLaunchKernelGGL((attn_partial_kernel<16, 2, 1, false, true, false, RULES>), grid, dim3(64), 0, st, A); break;
      case 3: hipLaunchKernelGGL((attn_partial_kernel<16, 3, 1, false, true, false, RULES>), grid, dim3(64), 0, st, A); break;
      default: hipLaunchKernelGGL((attn_partial_kernel<16, 4, 1, false, true, false, RULES>), grid, dim3(64), 0, st, A); break;
    }
    return;
  }
  switch (format_key(c)) {
    case 1602: launch_partial_g<16, 2, RULES>(A, G, lean, grid, st); break;
    case 1604: launch_partial_g<16, 4, RULES>(A, G, lean, grid, st); break;
    case 1608: launch_partial_g<16, 8, RULES>(A, G, lean, grid, st); break;
    case 802: launch_partial_g<8, 2, RULES>(A, G, lean, grid, st); break;
    case 1603: launch_partial_g<16, 3, RULES>(A, G, lean, grid, st); break;
    case 803: launch_partial_g<8, 3, RULES>(A, G, lean, grid, st); break;
    case 402: launch_partial_g<4, 2, RULES>(A, G, lean, grid, st); break;
    case 804: launch_partial_g<8, 4, RULES>(A, G, lean, grid, st); break;
    default: launch_partial_g<8, 8, RULES>(A, G, lean, grid, st); break;
  }
}

}  // namespace

}  // namespace mikv

#endif  // MIKV_ATTENTION_DEVICE_H
