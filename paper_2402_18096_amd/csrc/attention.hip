// Decode-step attention over the mixed-precision cache (Section 3.4, Fig. 3
// left) and the importance update (the H2O accumulated-attention score): the
// finalize kernels and the host side; the partial phase is in attention_device.h.
#include <algorithm>
#include <atomic>

#include "attention_device.h"
#include "select_device.h"

namespace mikv {

namespace {

// Softmax over the whole sequence from the chunk records (Section 2.1): a
// query head's max M is the largest chunk max, its normaliser L the chunk
// sums rescaled by exp2(m_r - M); the output is the rescaled value sums / L.
// Each block of the finalize kernel derives (M, 1/L) of the G query heads of
// KV head h from the (m, l) pairs, then turns one tile of scores into
// probabilities (and adds their GQA sum to the importance scores when
// asked); block 0 also merges the value sums into the output.
constexpr int kProbTile = 8 * kBlock;  // scores per block and query head

// (M, 1/L) of query heads qh0 .. qh0+G-1, computed by every wave on its own
// (no LDS, no barrier): lane r merges the (m, l) pairs of records r, r+64, ...
template <int G>
__device__ inline void head_stats(const AttnArgs &A, int qh0, int nc, float M[G], float inv[G]) {
  const int lane = threadIdx.x & 63;
  float m[G], l[G];
#pragma unroll
  for (int i = 0; i < G; ++i) {
    m[i] = kNegInf;
    l[i] = 0.0f;
  }
  for (int r = lane; r < nc; r += 64) {
    float2 ml[G];
#pragma unroll
    for (int i = 0; i < G; ++i)
      ml[i] = *reinterpret_cast<const float2 *>(A.partials + ((int64_t)(qh0 + i) * nc + r) * kRec);
#pragma unroll
    for (int i = 0; i < G; ++i) {
      if (ml[i].x > m[i]) {
        l[i] = fmaf(l[i], __builtin_amdgcn_exp2f(m[i] - ml[i].x), ml[i].y);
        m[i] = ml[i].x;
      } else if (ml[i].x != kNegInf) {
        l[i] = fmaf(ml[i].y, __builtin_amdgcn_exp2f(ml[i].x - m[i]), l[i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < G; ++i) {
    M[i] = wave_max(m[i]);
    const float total = wave_sum(m[i] == kNegInf ? 0.0f : l[i] * __builtin_amdgcn_exp2f(m[i] - M[i]));
    // a query that sees no token: probabilities and output 0
    if (M[i] == kNegInf) M[i] = 0.0f;
    inv[i] = total == 0.0f ? 0.0f : 1.0f / total;
  }
}

// One probability tile (kProbTile scores of every query head of KV head h):
// loaded first, so that the latency overlaps the statistics, then stored.
template <int G>
struct ProbTile {
  static constexpr int kPer = kProbTile / kBlock;
  float sv[kPer][G], a[kPer];
  int t[kPer];
  int n_pool;
};

// n_pool: the pool's token count (< 0: read the live counter).
template <int G>
__device__ inline ProbTile<G> prob_tile_load(const AttnArgs &A, int h, int qh0, bool is_hi, int tile, bool has_tile,
                                             bool accumulate, int n_pool = -1) {
  ProbTile<G> T;
  const int cap = is_hi ? A.cap_hi : A.cap_lo;
  const float *scores = is_hi ? A.scores_hi : A.scores_lo;
  const float *acc = is_hi && accumulate ? A.acc : nullptr;
#pragma unroll
  for (int u = 0; u < ProbTile<G>::kPer; ++u) {
    T.t[u] = tile * kProbTile + u * kBlock + threadIdx.x;
    const bool ok = has_tile && T.t[u] < cap;
#pragma unroll
    for (int i = 0; i < G; ++i)
      T.sv[u][i] = ok ? __builtin_nontemporal_load(&scores[(int64_t)(qh0 + i) * cap + T.t[u]]) : 0.0f;
    T.a[u] = ok && acc ? acc[(int64_t)h * A.cap_hi + T.t[u]] : 0.0f;
  }
  T.n_pool = !has_tile ? 0 : n_pool >= 0 ? n_pool : is_hi ? hi_count(A, h) : A.n_lo[h];
  return T;
}

// Probabilities of one tile, stored; with the importance update, the new
// score of every slot also goes to a_new[u] (the old one past the pool).
template <int G>
__device__ inline void prob_tile_store(const AttnArgs &A, int h, int qh0, bool is_hi, bool accumulate,
                                       const ProbTile<G> &T, const float M[G], const float inv[G],
                                       float *a_new = nullptr) {
  const int cap = is_hi ? A.cap_hi : A.cap_lo;
  float *probs = is_hi ? A.probs_hi : A.probs_lo;
  float *acc = is_hi && accumulate ? A.acc : nullptr;
#pragma unroll
  for (int u = 0; u < ProbTile<G>::kPer; ++u) {
    if (T.t[u] >= T.n_pool) {
      if (a_new) a_new[u] = T.a[u];
      continue;
    }
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < G; ++i) {
      const float p = __builtin_amdgcn_exp2f(T.sv[u][i] - M[i]) * inv[i];
      if (probs) __builtin_nontemporal_store(p, &probs[(int64_t)(qh0 + i) * cap + T.t[u]]);
      sum = i == 0 ? p : sum + p;
    }
    const float an = T.a[u] + sum;
    if (acc) acc[(int64_t)h * A.cap_hi + T.t[u]] = an;
    if (a_new) a_new[u] = an;
  }
}

// Output merge of the G query heads (whole block): thread -> (record split
// s, query head i, 4 channels q4), partial sums reduced in LDS.
template <int G>
__device__ inline void merge_output(const AttnArgs &A, int qh0, int nc, const float M[G], const float inv[G]) {
  constexpr int S = 8 / G;
  // Up to four query heads, a wave works on one head (i wave-uniform, so
  // picking its statistics is a scalar select, not a per-lane indexed array);
  // eight heads take two per wave.
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int q4 = lane & 31;
  const int i = G <= 4 ? __builtin_amdgcn_readfirstlane(wave % G) : (threadIdx.x / 32) % G;
  const int s = G <= 4 ? (wave / G) * 2 + (lane >> 5) : threadIdx.x / (32 * G);
  const float *rec = A.partials + (int64_t)(qh0 + i) * nc * kRec;
  // (through copies that the compiler cannot trace back to M and inv: it would
  // make indexed arrays of the choices, in scratch, or in LDS addressed
  // through the dispatch packet in host memory)
  float Mi = M[0], invi = inv[0];
#pragma unroll
  for (int j = 1; j < G; ++j) {
    float Mj = M[j], invj = inv[j];
    asm("" : "+v"(Mj), "+v"(invj));
    Mi = i == j ? Mj : Mi;
    invi = i == j ? invj : invi;
  }
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  // RB records per thread and batch, all loaded before any is used (a
  // missing record reads record 0 and gets weight 0): one memory round trip
  // per batch (a plain loop waits for every record in turn)
  constexpr int RB = 8;
  for (int r0 = s; r0 < nc; r0 += RB * S) {
    float mr[RB];
    float4 o[RB];
#pragma unroll
    for (int k = 0; k < RB; ++k) {
      const int r = r0 + k * S;
      const float *rr = rec + (int64_t)(r < nc ? r : 0) * kRec;
      mr[k] = r < nc ? rr[0] : kNegInf;
      o[k] = reinterpret_cast<const float4 *>(rr + kRecO)[q4];
    }
#pragma unroll
    for (int k = 0; k < RB; ++k) {
      const float w = mr[k] == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(mr[k] - Mi);
      v.x = fmaf(o[k].x, w, v.x);
      v.y = fmaf(o[k].y, w, v.y);
      v.z = fmaf(o[k].z, w, v.z);
      v.w = fmaf(o[k].w, w, v.w);
    }
  }
  __shared__ float4 s_o[kBlock];
  const int slot = (s * G + i) * 32 + q4;  // LDS by (split, head, channels)
  s_o[slot] = v;
  __syncthreads();
  if (s == 0) {
    for (int s2 = 1; s2 < S; ++s2) {
      const float4 u = s_o[slot + s2 * 32 * G];
      v.x += u.x;
      v.y += u.y;
      v.z += u.z;
      v.w += u.w;
    }
    reinterpret_cast<float4 *>(A.out + (int64_t)(qh0 + i) * kHeadDim)[q4] =
        make_float4(v.x * invi, v.y * invi, v.z * invi, v.w * invi);
  }
}

// Output merge of one KV head by `merges` blocks, this one `block`: one block
// for the group, or (merges = G) one per query head.
template <int G>
__device__ inline void merge_group(const AttnArgs &A, int qh0, int nc, int block, int merges) {
  if constexpr (G >= 4) {
    if (merges > 1) {
      float M[1], inv[1];
      head_stats<1>(A, qh0 + block, nc, M, inv);
      merge_output<1>(A, qh0 + block, nc, M, inv);
      return;
    }
  }
  float M[G], inv[G];
  head_stats<G>(A, qh0, nc, M, inv);
  merge_output<G>(A, qh0, nc, M, inv);
}

// Blocks (h, 0 .. merges - 1) merge the output of head h; the blocks after
// them turn one probability tile each into probabilities (importance-pool
// tiles first).  Heads run along x, so the longest blocks, the merges, are
// dispatched first.
// (Register budget: 8 blocks per CU for one query head per KV head, 6 for
// two; the grids of many-head caches hold several blocks per CU.)
template <int G>
__global__ __launch_bounds__(kBlock) __attribute__((amdgpu_waves_per_eu(G == 1 ? 8 : G == 2 ? 6 : 1)))
void attn_finalize_kernel(AttnArgs A, int accumulate, int tiles_hi, int tiles_lo, int per_query, int merges) {
  const int h = blockIdx.x, c = blockIdx.y;  // heads fastest: every head's merges are dispatched first
  const int qh0 = h * G;  // = b * q_heads + kv head * G
  const int nc = A.nc_hi + A.nc_lo;
  if constexpr (G < 4) merges = 1;  // (as merge_blocks has it, known to the compiler)
  if (c < merges) {  // a merge holds no tile
    merge_group<G>(A, qh0, nc, c, merges);
    return;
  }
  float M[G], inv[G];
  const int tile = c - merges;
  const bool is_hi = tile < tiles_hi;
  const bool has_tile = is_hi || tile - tiles_hi < tiles_lo;
  // With a block per query head of a group the pool's size is the one that
  // the partial phase noted in the record of its first chunk.
  const int n_pool = per_query ? __builtin_bit_cast(int, A.partials[((int64_t)qh0 * nc + (is_hi ? 0 : A.nc_hi)) * kRec + kRecN])
                               : -1;
  const ProbTile<G> T =
      prob_tile_load<G>(A, h, qh0, is_hi, is_hi ? tile : tile - tiles_hi, has_tile, accumulate, n_pool);
  head_stats<G>(A, qh0, nc, M, inv);
  if (has_tile) prob_tile_store<G>(A, h, qh0, is_hi, accumulate, T, M, inv);
}

// Finalize with the importance update and the re-rank fused (the decode
// step).  Block (h, 0) of head h turns every importance-pool tile into
// probabilities and new scores and, its own writes being the only scores
// the re-rank reads, runs the head's top-k and demotion on the scores it
// still holds in registers (the positions and the last slot are loaded
// with the tiles, so the re-rank adds one memory round trip: the demoted
// row).  Blocks (h, 1 .. merges) merge the output: one block for the group, or
// one per query head (merge_blocks); the blocks after them handle the
// retained-pool tiles.  Heads run along x, so every head's re-rank block is
// dispatched before any tile block.  No block waits on another.
#ifndef MIKV_LO_TILES
#define MIKV_LO_TILES 8
#endif
// Retained-pool probability tiles per finalize block (a tile per query head
// of the group costs the same registers as G tiles of one head):
// MIKV_LO_TILES / G, except 4 at G = 4, where the fewer, longer blocks (216
// registers, two waves per SIMD) finish the step sooner than 2 or 1 tiles
// per block (8 is slower again).
#ifndef MIKV_LO_TILES_G4
#define MIKV_LO_TILES_G4 4
#endif
__host__ __device__ constexpr int lo_tiles_per_block(int G) {
  return G == 4 ? MIKV_LO_TILES_G4 : MIKV_LO_TILES / G > 1 ? MIKV_LO_TILES / G : 1;
}

template <int G, int HI, int LO>
__global__ __launch_bounds__(kBlock) void finalize_select_kernel(AttnArgs A, int tiles_hi, int tiles_lo, int merges, SelArgs S) {
  static_assert(kSel == kBlock && kSelItems * kBlock == 2 * kProbTile, "select items = two probability tiles");
  const int h = blockIdx.x, c = blockIdx.y;  // heads fastest: every head's block 0 is dispatched first
  const int b = h / A.kv_heads, kvh = h % A.kv_heads;
  const int qh0 = b * A.q_heads + kvh * G;
  const int nc = A.nc_hi + A.nc_lo;
  if constexpr (G < 4) merges = 1;  // (as merge_blocks has it, known to the compiler)
  if (c >= 1 && c <= merges) {  // a merge holds no tile
    merge_group<G>(A, qh0, nc, c - 1, merges);
    return;
  }
  if (c > merges) {
    // kLoTiles retained-pool tiles per block, all loaded before the
    // statistics: fewer, longer blocks (one round of blocks per step).
    // Block (h, 0) raises n_lo when it demotes, concurrently with this
    // block, so the retained pool's size at attention time comes from the
    // record of the head's first retained-pool chunk, written by the
    // partial phase.
    constexpr int KT = lo_tiles_per_block(G);
    const int t0 = (c - 1 - merges) * KT;
    const int n_lo_att = __builtin_bit_cast(
        int, A.partials[((int64_t)qh0 * nc + A.nc_hi) * kRec + kRecN]);
    ProbTile<G> T[KT];
#pragma unroll
    for (int k = 0; k < KT; ++k)
      T[k] = prob_tile_load<G>(A, h, qh0, false, t0 + k, t0 + k < tiles_lo, false, n_lo_att);
    float M[G], inv[G];
    head_stats<G>(A, qh0, nc, M, inv);
#pragma unroll
    for (int k = 0; k < KT; ++k)
      if (t0 + k < tiles_lo) prob_tile_store<G>(A, h, qh0, false, false, T[k], M, inv);
    return;
  }
  // Everything the re-rank reads besides the new scores is loaded together
  // with the first two tiles and the chunk statistics.
  const int n = __builtin_amdgcn_readfirstlane(hi_count(A, h));
  const int n_lo0 = __builtin_amdgcn_readfirstlane(S.n_lo[h]);
  const int thr = S.length - S.window;  // positions >= thr are in the window
  // two tiles in flight for one or two query heads per KV head; with more,
  // the second waits for the statistics (the block's register budget also
  // bounds the occupancy of the retained-pool tile blocks)
  constexpr bool kTwoAhead = G <= 2;
  const ProbTile<G> T0 = prob_tile_load<G>(A, h, qh0, true, 0, tiles_hi > 0, true);
  ProbTile<G> T1;
  if constexpr (kTwoAhead) T1 = prob_tile_load<G>(A, h, qh0, true, 1, tiles_hi > 1, true);
  int pv[kSelItems];
  const int32_t *pos = S.hi_pos + (int64_t)h * S.cap_hi;
#pragma unroll
  for (int u = 0; u < kSelItems; ++u) {
    const int i = u * kSel + threadIdx.x;
    pv[u] = i < S.cap_hi ? pos[i] : thr;
  }
  SlotData<HI> last = n > 0 ? load_slot<HI>(S, h, n - 1) : SlotData<HI>{};
  float M[G], inv[G];
  head_stats<G>(A, qh0, nc, M, inv);
  float an[kSelItems];
  prob_tile_store<G>(A, h, qh0, true, true, T0, M, inv, an);
  if constexpr (!kTwoAhead) T1 = prob_tile_load<G>(A, h, qh0, true, 1, tiles_hi > 1, true);
  prob_tile_store<G>(A, h, qh0, true, true, T1, M, inv, an + ProbTile<G>::kPer);
  for (int tile = 2; tile < tiles_hi; ++tile) {
    const ProbTile<G> T = prob_tile_load<G>(A, h, qh0, true, tile, true, true);
    prob_tile_store<G>(A, h, qh0, true, true, T, M, inv);
  }
  // slot u * kSel + t of thread t is item u of the two first tiles
  SelScan sc;
  __shared__ float s_last;
#pragma unroll
  for (int u = 0; u < kSelItems; ++u) {
    const int i = u * kSel + threadIdx.x;
    if (i < n && pv[u] < thr) sc.add(i, pv[u], an[u]);
    if (i == n - 1) s_last = an[u];
  }
  // slots past the first two tiles: from memory, written above by this same thread
  if (S.cap_hi > kSel * kSelItems) select_scan(S, h, kSel * kSelItems, n, thr, sc);
  __syncthreads();  // the block's score updates (and s_last) are complete before the re-rank uses them
  if (threadIdx.x == 0 && n > 0)
    last.acc = n - 1 < kSel * kSelItems ? s_last : S.hi_acc[(int64_t)h * S.cap_hi + n - 1];
  select_finish<HI, LO>(S, h, n, n_lo0, sc, last, A.hi_pending != 0);
}

template <int G>
__global__ __launch_bounds__(kBlock) void importance_kernel(float *acc, const float *probs, const int32_t *n_hi,
                                                            int cap_hi, int q_heads, int kv_heads) {
  const int h = blockIdx.y;
  const int t = blockIdx.x * kBlock + threadIdx.x;
  if (t >= n_hi[h]) return;
  const int b = h / kv_heads, kvh = h % kv_heads;
  const int qh0 = b * q_heads + kvh * G;
  float sum = probs[(int64_t)qh0 * cap_hi + t];
#pragma unroll
  for (int i = 1; i < G; ++i) sum = sum + probs[(int64_t)(qh0 + i) * cap_hi + t];
  acc[(int64_t)h * cap_hi + t] += sum;
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
struct Plan {
  int chunk_hi, chunk_lo, nc_hi, nc_lo;
  int nc_first;  // nc_hi + the retained-pool chunks that hold tokens whatever the split
  int64_t head_bytes_hi, head_bytes_lo;  // packed bytes of one head's occupied span per pool (upper bound)
};

int round_up(int64_t x, int m) { return (int)(((x + m - 1) / m) * m); }

// The resident share (mikv_set_resident_bytes): bytes of a cache read with
// plain loads.
std::atomic<int64_t> g_resident_bytes{kResidentBytes};
int64_t resident_budget() { return g_resident_bytes.load(std::memory_order_relaxed); }

size_t workspace_bytes_for(const mikv_cache *c, const Plan &p) {
  const int64_t BQ = (int64_t)c->batch * c->q_heads;
  return (size_t)(BQ * (p.nc_hi + p.nc_lo) * kRec * 4 + BQ * c->cap_hi * 4);
}

constexpr int64_t kSimds = 1024, kFewWaves = 2 * kSimds;
constexpr size_t kFewWorkspace = (size_t)16 << 20;

// size_bound: the plan with the most chunks the resident share can give, and
// without the shorter chunks of few waves (workspace_need sizes workspaces
// from it, so a workspace stays large enough when the share changes).
Plan make_plan(const mikv_cache *c, int length, bool size_bound = false) {
  Plan p;
  const int64_t NH = n_heads_of(c);
  // an evicting cache has no retained pool: no chunks for it
  const int span_hi = std::min(length, c->cap_hi), span_lo = evicting(c) ? 0 : std::min(length, c->cap_lo);
  const int64_t bh = token_bytes(c->hi_bits, c->group), bl = token_bytes(evicting(c) ? 2 : c->lo_bits, c->group);
  const int64_t total = NH * (span_hi * bh + span_lo * bl);
  p.head_bytes_hi = span_hi * bh;
  p.head_bytes_lo = span_lo * bl;
  // One wave per chunk; up to 64 KiB (MHA) or 96 KiB (GQA) of packed K/V per
  // chunk (many small work units balance the CUs best), at least 16 KiB so
  // the per-chunk merge stays cheap.  Chunks are whole wave iterations (128
  // tokens).
  const int64_t chunk_kb = group_size_of(c) == 1 ? MIKV_CHUNK_KB_MHA : MIKV_CHUNK_KB;
  int64_t target = std::max<int64_t>(std::min<int64_t>(total / 4096, chunk_kb << 10), 16 << 10);
  const int cmax = max_chunk(group_size_of(c));
  // MHA importance-pool rows cost the least work per byte: more bytes per
  // chunk there cut the per-wave overhead (twice: 4 % of the long_context
  // step).  Four times pays only for an fp16 pool read from the last-level
  // cache (the whole pool within the resident share: long_context warm
  // 1.3 % faster); streamed from HBM those longer waves were slower (cold
  // step 130 -> 134 us), and an INT8 pool lost 2.6 % at the 13B shape.
  // GQA rows carry G queries' work and keep one share.
  const bool hi_resident = !size_bound && NH * p.head_bytes_hi <= resident_budget();
  const int64_t hi_scale = c->hi_bits == 16 && hi_resident ? MIKV_CHUNK_HI_SCALE_F16 : MIKV_CHUNK_HI_SCALE;
  const int64_t target_hi = group_size_of(c) == 1 ? target * hi_scale : target;
  p.chunk_hi = std::min(cmax, std::max(128, round_up(target_hi / bh, 128)));
  p.chunk_lo = std::min(cmax, std::max(128, round_up(target / bl, 128)));
  auto chunks = [&]() {
    p.nc_hi = std::max(1, (span_hi + p.chunk_hi - 1) / p.chunk_hi);
    p.nc_lo = evicting(c) ? 0 : std::max(1, (span_lo + p.chunk_lo - 1) / p.chunk_lo);
  };
  chunks();
  // From four query heads per KV head on, a wave takes two (G = 8: four) times
  // as many iterations for an importance-pool chunk as for a retained-pool one,
  // and while the waves all fit the chip at once the longest of them is the
  // launch.  Then shorter chunks: retained pool 128 tokens while twice the
  // waves still fit, importance pool down to 32 as long as they do.  What fits:
  // at G = 8 two waves per SIMD; at G = 4, whose chunks are half as long, one
  // while the long chunks leave SIMDs idle (two that share a SIMD take longer
  // than the long chunk did: 2 x 32/8 heads x 8000 tokens, balanced fp16 + INT2,
  // 18.9 us per attention in long chunks, 17.2 with one per SIMD, 19.6 with
  // two; 14 x 32/8 x 710, INT8 + INT4, 18.3, 18.7, 24.2), and two when the long
  // chunks already share them, where shorter ones even out the load (4 x 32/8 x
  // 8192, INT8 + INT2, 23.0 -> 20.8), except for fp16 + INT2, where they only
  // add records (2 x 32/8 x 12000 19.3 -> 20.2, balanced 20.5 -> 23.7).
  // Measured (us per attention, long -> short): 1 sequence x 64/8 heads x 4096
  // tokens 29.9 -> 16.0, 4 x 64/8 x 7001 46.1 -> 28.1, 1 x 32/8 x 4096 14.6 ->
  // 11.4, 4 x 32/8 x 4096 17.1 -> 16.0; with one query head shorter chunks gain
  // nothing (1 x 40 x 5003: 15.2 -> 16.6).  The whole step, whose merge reads
  // the records (merge_blocks): 39.2 -> 26.1, 56.6 -> 38.3, 22.3 -> 18.9, 26.6
  // -> 23.3; 1 x 32/4 x 32768 (464 records) 55.9 -> 51.4.
  const int64_t base = NH * (p.nc_hi + p.nc_lo);
  const int G = group_size_of(c);
  // With codes in both pools and 3 bits or more in the retained one (at G = 8,
  // where a wave has the most arithmetic, also for fp16 + INT4 and INT8) two waves that
  // share a SIMD always lose: one while the long chunks leave SIMDs idle (at G = 8
  // three to four SIMDs, since a full one doubles some), else the long
  // chunks (us with the importance update, long, two waves, this: 4 x 64/8 x
  // 4000, INT8 + INT3 40.3, 51.7, 38.6; 4 x 32/8 x 4000 24.8, 28.5, 22.3).
  const bool arith = c->lo_bits != 2 && (c->hi_bits != 16 || (G >= 8 && c->lo_bits >= 4));
  const int64_t one = G >= 8 ? kSimds * 3 / 4 : kSimds;
  const int64_t fit = G < 4 || base >= kFewWaves            ? 0
                      : arith                               ? (base < one ? one : 0)
                      : G >= 8                              ? kFewWaves
                      : base < kSimds                       ? kSimds
                      : c->hi_bits == 16 && c->lo_bits == 2 ? 0
                                                            : kFewWaves;
  if (!size_bound && fit) {
    const Plan wide = p;
    if (2 * base <= fit && p.nc_lo) p.chunk_lo = std::min(p.chunk_lo, 128);
    const int step = c->hi_bits == 4 ? 32 : 16;  // whole iterations
    for (p.chunk_hi = 32;; p.chunk_hi += step) {
      chunks();
      if (p.chunk_hi >= wide.chunk_hi || NH * (p.nc_hi + p.nc_lo) <= fit) break;
    }
    // (a workspace that a caller's scratch of a fixed size held before still does)
    if (NH * (p.nc_hi + p.nc_lo) > fit || workspace_bytes_for(c, p) > kFewWorkspace) p = wide;
  }
  // every token is in one of the pools, so at least length - cap_hi are in
  // the retained one (only the dispatch order depends on this)
  const int lo_min = std::max(0, std::min(span_lo, length - c->cap_hi));
  p.nc_first = p.nc_hi + std::min(p.nc_lo, (lo_min + p.chunk_lo - 1) / p.chunk_lo);
  return p;
}

// Blocks that merge the output of one KV head's group where the finalize
// updates the importance (in both of its kernels, so that the decode step
// and the separate calls agree bit for bit).  One block holds S = 8 / G splits of the records for each of the G
// query heads, so at G = 8 it reads them all in turn, eight per round trip:
// with the records of short chunks (or of few long-context heads) it outlasts
// the rest of the launch (us per step, one block -> G: 1 x 32/4 heads x 32768
// tokens, 464 records, 69.4 -> 51.6; 1 x 16/2 x 32768 65.2 -> 46.7; 23 x 32/8 x
// 1113 36.1 -> 27.2).  A block per query head has eight splits.  With more waves
// than fit the chip the merges of many heads share it and G blocks each read
// the statistics for nothing: mistral_7b (5120 waves) 2 % slower.
int merge_blocks(const mikv_cache *c, const Plan &p) {
  const int G = group_size_of(c);
  return G >= 4 && n_heads_of(c) * (int64_t)(p.nc_hi + p.nc_lo) <= kFewWaves ? G : 1;
}

// Bytes of workspace for `length` tokens.  From four query heads per KV head
// on a shorter length can have the more chunks (the shorter ones of few
// waves), and a workspace made for a generation's last length serves all of
// it: so the most records that such chunks can have at this or any shorter
// length count (they are at least 32 and 128 tokens long and at most kFewWaves,
// in at most kFewWorkspace bytes).
size_t workspace_need(const mikv_cache *c, int length) {
  const Plan p = make_plan(c, length, true);
  const size_t need = workspace_bytes_for(c, p);
  if (group_size_of(c) < 4) return need;
  const int span_hi = std::min(length, c->cap_hi), span_lo = evicting(c) ? 0 : std::min(length, c->cap_lo);
  Plan few = p;
  few.nc_hi = (int)std::min<int64_t>(kFewWaves / n_heads_of(c), (span_hi + 31) / 32 + (span_lo + 127) / 128 + 1);
  few.nc_lo = 0;
  return std::max(need, std::min(workspace_bytes_for(c, few), kFewWorkspace));
}

AttnArgs make_args(const mikv_cache *c, const Plan &p, const uint16_t *q, const float *balance, float scale,
                   float *out, float *probs_hi, float *probs_lo, int flags, void *ws) {
  AttnArgs A;
  A.hi_k = (const uint8_t *)c->hi_k;
  A.hi_v = (const uint8_t *)c->hi_v;
  A.hi_kp = (const uint32_t *)c->hi_kp;
  A.hi_vp = (const uint32_t *)c->hi_vp;
  A.n_hi = c->n_hi;
  A.lo_k = c->lo_k;
  A.lo_v = c->lo_v;
  A.lo_kp = (const uint32_t *)c->lo_kp;
  A.lo_vp = (const uint32_t *)c->lo_vp;
  A.n_lo = c->n_lo;
  A.q = q;
  A.balance = balance;
  A.scale = scale;
  const int64_t BQ = (int64_t)c->batch * c->q_heads;
  A.partials = (float *)ws;
  float *ws_scores = A.partials + BQ * (p.nc_hi + p.nc_lo) * kRec;
  const bool acc = (flags & MIKV_ATTN_ACCUMULATE) != 0;
  A.scores_hi = probs_hi ? probs_hi : (acc ? ws_scores : nullptr);
  A.scores_lo = probs_lo;
  A.probs_hi = probs_hi;
  A.probs_lo = probs_lo;
  A.acc = acc ? c->hi_acc : nullptr;
  A.out = out;
  A.cap_hi = c->cap_hi;
  A.cap_lo = c->cap_lo;
  A.group = c->group;
  A.q_heads = c->q_heads;
  A.kv_heads = c->kv_heads;
  A.chunk_hi = p.chunk_hi;
  A.chunk_lo = p.chunk_lo;
  A.nc_hi = p.nc_hi;
  A.nc_lo = p.nc_lo;
  A.nc_first = p.nc_first;
  A.app = AppendArgs{};
  A.hi_pending = 0;
  // fp16 importance-pool chunks under GQA run longest: dispatched first, the
  // tail of the grid is shorter (measured: mistral_7b 66.0 -> 64.7 us per
  // launch).  With one query head per KV head the resident importance-pool
  // rows (last-level cache) and the streamed retained-pool rows (HBM) are
  // best read side by side, head by head (long_context 98.2 -> 95.0 us).
  A.pool_major = c->hi_bits == 16 && group_size_of(c) > 1 ? 1 : 0;
  A.order = 0;
  // Rows read plainly: up to resident_budget() bytes of the cache,
  // importance pool first (it is read by every step whatever the re-rank
  // does), then retained-pool heads.
  {
    const int64_t NH = n_heads_of(c);
    int64_t budget = resident_budget();
    const int64_t hb = std::max<int64_t>(p.head_bytes_hi, 1), lb = std::max<int64_t>(p.head_bytes_lo, 1);
    A.res_hi = (int)std::min<int64_t>(NH, budget / hb);
    budget -= (int64_t)A.res_hi * p.head_bytes_hi;
    A.res_lo = A.res_hi == NH ? (int)std::min<int64_t>(NH, budget / lb) : 0;
  }
  A.lo_kb = c->key_block ? (const uint32_t *)c->lo_kb : nullptr;
  A.hi_pos = c->hi_pos;
  A.lo_pos = c->lo_pos;
  A.rules = RuleArgs{};
  A.n_kblk = c->key_block ? key_blocks_of(c) : 0;
  return A;
}

// The fold of the decode step's append into the attention (position
// length - 1).
void set_append(AttnArgs &A, const mikv_cache *c, int32_t length, const uint16_t *k_new, const uint16_t *v_new,
                const float *balance) {
  AppendArgs &a = A.app;
  a.hi_k = (uint8_t *)c->hi_k;
  a.hi_v = (uint8_t *)c->hi_v;
  a.hi_kp = (uint32_t *)c->hi_kp;
  a.hi_vp = (uint32_t *)c->hi_vp;
  a.hi_pos = c->hi_pos;
  a.hi_acc = c->hi_acc;
  a.map = c->map;
  a.status = c->status;
  a.k = k_new;
  a.v = v_new;
  a.balance = balance;
  a.score_init = nullptr;
  a.cap_hi = c->cap_hi;
  a.max_len = c->max_len;
  a.group = c->group;
  a.pos = length - 1;
  A.hi_pending = 1;
}

// Whether an INT4 retained pool takes its rows two tiles at a time (unroll_lo):
// while at least half of the cache is read from the last-level cache.  Measured
// (us per attention, four tiles -> two): 8 x 32 heads x 4096 tokens, INT8 + INT4,
// 229 MB 38.2 -> 36.9; 16 x 32 x 2000 40.8 -> 39.4; 2 x 32 x 32768, 397 MB 69.0 ->
// 68.1; but mostly streamed, where bytes in flight count, 16 x 32 x 8192, fp16 +
// INT4, 905 MB 139.5 -> 142.3; 32 x 40 x 8192, INT8 + INT4, 2.3 GB 364 -> 375.
bool partial_lean(const mikv_cache *c, const Plan &p) {
  return n_heads_of(c) * (p.head_bytes_hi + p.head_bytes_lo) <= 2 * resident_budget();
}

int check_attention_args(const mikv_cache *c, int32_t length, const uint16_t *q, const float *balance, float *out,
                         void *ws, size_t ws_bytes, const char *who) {
  int rc = validate_cache(c);
  if (rc) return rc;
  if (!q || !out) return set_error(MIKV_ERR_INVALID_ARG, "%s: q/out is NULL", who);
  if (((uintptr_t)q | (uintptr_t)balance) % 16 != 0)
    return set_error(MIKV_ERR_INVALID_ARG, "%s: q and balance must be 16-byte aligned", who);
  if (length < 1) return set_error(MIKV_ERR_INVALID_ARG, "%s: length must be >= 1", who);
  if (length > c->max_len) return set_error(MIKV_ERR_CAPACITY, "%s: length %d > max_len %d", who, length, c->max_len);
  size_t need = workspace_need(c, length);
  if (!ws || ws_bytes < need) return set_error(MIKV_ERR_CAPACITY, "%s: workspace too small (%zu < %zu)", who, ws_bytes, need);
  return MIKV_OK;
}

}  // namespace

}  // namespace mikv

using namespace mikv;

extern "C" size_t mikv_decode_workspace_size(const mikv_cache *c, int32_t length) {
  if (!c || length < 1 || validate_cache(c)) return 0;
  return workspace_need(c, length);
}

namespace mikv {

int check_cap(float cap, float scale, const char *who) {
  if (!(cap >= 0.0f) || cap == __builtin_huge_valf())
    return set_error(MIKV_ERR_INVALID_ARG, "%s: cap must be >= 0 and finite", who);
  if (cap > 0.0f && scale / cap < 0x1p-126f)
    return set_error(MIKV_ERR_INVALID_ARG, "%s: scale / cap is below the fp32 range", who);
  return MIKV_OK;
}

int check_decode_rules(const mikv_score_rules *r, float scale, const char *who) {
  if (!r) return MIKV_OK;
  if (int e = check_cap(r->cap, scale, who)) return e;
  if (r->end) return set_error(MIKV_ERR_INVALID_ARG, "%s: a decode step takes no end", who);
  if (r->window < 0) return set_error(MIKV_ERR_INVALID_ARG, "%s: window must be >= 0", who);
  if (((uintptr_t)r->slopes | (uintptr_t)r->begin) % 4)
    return set_error(MIKV_ERR_INVALID_ARG, "%s: misaligned rules", who);
  return MIKV_OK;
}

int decode_partial(const mikv_cache *c, int32_t length, const uint16_t *q, const float *balance, float scale,
                   float *out, float *probs_hi, float *probs_lo, int32_t flags, void *ws, size_t ws_bytes,
                   const uint16_t *k_new, const uint16_t *v_new, const mikv_score_rules *rules, hipStream_t st) {
  int rc = check_attention_args(c, length, q, balance, out, ws, ws_bytes, "mikv_decode_attention_partial");
  if (rc) return rc;
  Plan p = make_plan(c, length);
  AttnArgs A = make_args(c, p, q, balance, scale, out, probs_hi, probs_lo, flags, ws);
  if (k_new) set_append(A, c, length, k_new, v_new, balance);
  // Odd lengths run the grid backwards, so consecutive decode steps read the
  // cache in opposite orders and each starts on what the 256 MB last-level
  // cache kept from the one before.  Wholly backwards with an fp16 importance
  // pool and one query head per KV head; under GQA or with an INT8 pool only
  // the head order flips, which keeps the longest waves at the front
  // (measured per step: long_context 136.4 -> 123.7 us wholly, 132.2 heads
  // only; mistral_7b 89.5 -> 87.0 heads only, 88.3 wholly; llama2_13b 335.7
  // -> 329.2 heads only; llama2_7b, whose cache fits that cache, unchanged).
  if (length & 1) A.order = c->hi_bits == 16 && group_size_of(c) == 1 ? 2 : 1;
  const dim3 grid((p.nc_hi + p.nc_lo) * n_heads_of(c));
  const bool lean = partial_lean(c, p);
  if (c->key_block && balance)
    return set_error(MIKV_ERR_INVALID_ARG, "mikv_decode_attention: per-channel keys take no balancer");
  if (rules && (rules->cap > 0.0f || rules->slopes || rules->begin || rules->window > 0)) {
    A.rules.cap = rules->cap * kLog2e;
    A.rules.cap_scale = rules->cap > 0.0f ? scale / rules->cap : 0.0f;
    A.rules.slopes = rules->slopes;
    A.rules.begin = rules->begin;
    A.rules.last = length - 1;
    A.rules.window = rules->window;
    launch_partial_rules(A, c, lean, grid, st);
  } else {
    launch_partial_c<false>(A, c, lean, grid, st);
  }
  return check_launch("mikv_decode_attention_partial");
}

template <int HI, int LO>
void launch_finalize_select(const AttnArgs &A, const SelArgs &S, int G, dim3 grid, int tiles_hi, int tiles_lo,
                            int merges, hipStream_t st) {
  switch (G) {
    case 1: hipLaunchKernelGGL((finalize_select_kernel<1, HI, LO>), grid, dim3(kBlock), 0, st, A, tiles_hi, tiles_lo, merges, S); break;
    case 2: hipLaunchKernelGGL((finalize_select_kernel<2, HI, LO>), grid, dim3(kBlock), 0, st, A, tiles_hi, tiles_lo, merges, S); break;
    case 4: hipLaunchKernelGGL((finalize_select_kernel<4, HI, LO>), grid, dim3(kBlock), 0, st, A, tiles_hi, tiles_lo, merges, S); break;
    default: hipLaunchKernelGGL((finalize_select_kernel<8, HI, LO>), grid, dim3(kBlock), 0, st, A, tiles_hi, tiles_lo, merges, S); break;
  }
}

int decode_finalize_select(const mikv_cache *c, int32_t length, const uint16_t *q, const float *balance, float scale,
                           float *out, float *probs_hi, float *probs_lo, void *ws, size_t ws_bytes, int32_t k_heavy,
                           int32_t window, void *sel_ws, bool appended, hipStream_t st) {
  int rc = check_attention_args(c, length, q, balance, out, ws, ws_bytes, "mikv_decode_step");
  if (rc) return rc;
  Plan p = make_plan(c, length);
  AttnArgs A = make_args(c, p, q, balance, scale, out, probs_hi, probs_lo, MIKV_ATTN_ACCUMULATE, ws);
  A.hi_pending = appended ? 1 : 0;
  const SelArgs S = make_sel_args(c, length, k_heavy, window, sel_ws);
  const int span_hi = std::min(length, c->cap_hi), span_lo = std::min(length, c->cap_lo);
  const int tiles_hi = (span_hi + kProbTile - 1) / kProbTile;  // probabilities accumulated
  const int tiles_lo = A.probs_lo && !evicting(c) ? (span_lo + kProbTile - 1) / kProbTile : 0;
  const int kt = lo_tiles_per_block(group_size_of(c));
  const int G = group_size_of(c);
  const int merges = merge_blocks(c, p);
  // y = 0: importance pool and re-rank, 1 .. merges: output
  dim3 grid(n_heads_of(c), 1 + merges + (tiles_lo + kt - 1) / kt);
  switch (format_key(c)) {
    case 1602: launch_finalize_select<16, 2>(A, S, G, grid, tiles_hi, tiles_lo, merges, st); break;
    case 1604: launch_finalize_select<16, 4>(A, S, G, grid, tiles_hi, tiles_lo, merges, st); break;
    case 1608: launch_finalize_select<16, 8>(A, S, G, grid, tiles_hi, tiles_lo, merges, st); break;
    case 802: launch_finalize_select<8, 2>(A, S, G, grid, tiles_hi, tiles_lo, merges, st); break;
    case 1603: launch_finalize_select<16, 3>(A, S, G, grid, tiles_hi, tiles_lo, merges, st); break;
    case 803: launch_finalize_select<8, 3>(A, S, G, grid, tiles_hi, tiles_lo, merges, st); break;
    case 402: launch_finalize_select<4, 2>(A, S, G, grid, tiles_hi, tiles_lo, merges, st); break;
    case 804: launch_finalize_select<8, 4>(A, S, G, grid, tiles_hi, tiles_lo, merges, st); break;
    default: launch_finalize_select<8, 8>(A, S, G, grid, tiles_hi, tiles_lo, merges, st); break;
  }
  return check_launch("mikv_decode_step (finalize and select)");
}

}  // namespace mikv

extern "C" int mikv_decode_attention_partial(const mikv_cache *c, int32_t length, const uint16_t *q,
                                             const float *balance, float scale, float *out, float *probs_hi,
                                             float *probs_lo, int32_t flags, void *ws, size_t ws_bytes,
                                             void *stream) {
  return decode_partial(c, length, q, balance, scale, out, probs_hi, probs_lo, flags, ws, ws_bytes, nullptr, nullptr,
                        nullptr, (hipStream_t)stream);
}

namespace mikv {

int decode_finalize(const mikv_cache *c, int32_t length, const uint16_t *q, const float *balance, float scale,
                    float *out, float *probs_hi, float *probs_lo, int32_t flags, void *ws, size_t ws_bytes,
                    bool appended, hipStream_t st) {
  int rc = check_attention_args(c, length, q, balance, out, ws, ws_bytes, "mikv_decode_attention_finalize");
  if (rc) return rc;
  Plan p = make_plan(c, length);
  AttnArgs A = make_args(c, p, q, balance, scale, out, probs_hi, probs_lo, flags, ws);
  A.hi_pending = appended ? 1 : 0;
  const int acc = (flags & MIKV_ATTN_ACCUMULATE) ? 1 : 0;
  // probability tiles: importance pool when its probabilities are emitted or
  // accumulated, retained pool when its probabilities are emitted
  const int span_hi = std::min(length, c->cap_hi), span_lo = std::min(length, c->cap_lo);
  const int tiles_hi = (A.scores_hi && (A.probs_hi || A.acc)) ? (span_hi + kProbTile - 1) / kProbTile : 0;
  const int tiles_lo = A.probs_lo && !evicting(c) ? (span_lo + kProbTile - 1) / kProbTile : 0;
  // Without the importance update nothing is summed over the query heads of a
  // KV head: each is a head of its own then, in G times the blocks of a G-th of
  // the work (finalize of 4 x 64/8 x 7001 tokens 10.1 -> 5.3 us, of 16 x
  // 64/8 x 8192 5 us less; MHA as before).
  const int G = acc ? group_size_of(c) : 1, per_query = G != group_size_of(c);
  const int merges = per_query ? 1 : merge_blocks(c, p);
  dim3 grid(c->batch * c->q_heads / G, merges + tiles_hi + tiles_lo);  // y < merges: output
  switch (G) {
    case 1: hipLaunchKernelGGL(attn_finalize_kernel<1>, grid, dim3(kBlock), 0, st, A, acc, tiles_hi, tiles_lo, per_query, merges); break;
    case 2: hipLaunchKernelGGL(attn_finalize_kernel<2>, grid, dim3(kBlock), 0, st, A, acc, tiles_hi, tiles_lo, per_query, merges); break;
    case 4: hipLaunchKernelGGL(attn_finalize_kernel<4>, grid, dim3(kBlock), 0, st, A, acc, tiles_hi, tiles_lo, per_query, merges); break;
    default: hipLaunchKernelGGL(attn_finalize_kernel<8>, grid, dim3(kBlock), 0, st, A, acc, tiles_hi, tiles_lo, per_query, merges); break;
  }
  return check_launch("mikv_decode_attention_finalize");
}

}  // namespace mikv

extern "C" int mikv_decode_attention_finalize(const mikv_cache *c, int32_t length, const uint16_t *q,
                                              const float *balance, float scale, float *out, float *probs_hi,
                                              float *probs_lo, int32_t flags, void *ws, size_t ws_bytes,
                                              void *stream) {
  return decode_finalize(c, length, q, balance, scale, out, probs_hi, probs_lo, flags, ws, ws_bytes, false,
                         (hipStream_t)stream);
}

extern "C" int mikv_decode_attention(const mikv_cache *c, int32_t length, const uint16_t *q, const float *balance,
                                     float scale, float *out, float *probs_hi, float *probs_lo, int32_t flags,
                                     void *ws, size_t ws_bytes, void *stream) {
  int rc = mikv_decode_attention_partial(c, length, q, balance, scale, out, probs_hi, probs_lo, flags, ws,
                                         ws_bytes, stream);
  if (rc) return rc;
  return mikv_decode_attention_finalize(c, length, q, balance, scale, out, probs_hi, probs_lo, flags, ws,
                                        ws_bytes, stream);
}

extern "C" int mikv_decode_attention_scored(const mikv_cache *c, int32_t length, const uint16_t *q, const float *balance,
                                            float scale, const mikv_score_rules *rules, float *out, float *probs_hi,
                                            float *probs_lo, int32_t flags, void *ws, size_t ws_bytes, void *stream) {
  int rc = check_decode_rules(rules, scale, "mikv_decode_attention_scored");
  if (rc) return rc;
  rc = decode_partial(c, length, q, balance, scale, out, probs_hi, probs_lo, flags, ws, ws_bytes, nullptr, nullptr, rules,
                      (hipStream_t)stream);
  if (rc) return rc;
  return decode_finalize(c, length, q, balance, scale, out, probs_hi, probs_lo, flags, ws, ws_bytes, false,
                         (hipStream_t)stream);
}

extern "C" int mikv_importance_update(const mikv_cache *c, int32_t length, const float *probs_hi, void *stream) {
  int rc = validate_cache(c);
  if (rc) return rc;
  if (!probs_hi) return set_error(MIKV_ERR_INVALID_ARG, "mikv_importance_update: probs_hi is NULL");
  if (length < 1 || length > c->max_len)
    return set_error(length < 1 ? MIKV_ERR_INVALID_ARG : MIKV_ERR_CAPACITY,
                     "mikv_importance_update: length %d outside [1, max_len]", length);
  const int span = std::min(length, c->cap_hi);
  dim3 grid((span + kBlock - 1) / kBlock, n_heads_of(c));
  hipStream_t st = (hipStream_t)stream;
  switch (group_size_of(c)) {
    case 1:
      hipLaunchKernelGGL(importance_kernel<1>, grid, dim3(kBlock), 0, st, c->hi_acc, probs_hi, c->n_hi, c->cap_hi,
                         c->q_heads, c->kv_heads);
      break;
    case 2:
      hipLaunchKernelGGL(importance_kernel<2>, grid, dim3(kBlock), 0, st, c->hi_acc, probs_hi, c->n_hi, c->cap_hi,
                         c->q_heads, c->kv_heads);
      break;
    case 4:
      hipLaunchKernelGGL(importance_kernel<4>, grid, dim3(kBlock), 0, st, c->hi_acc, probs_hi, c->n_hi, c->cap_hi,
                         c->q_heads, c->kv_heads);
      break;
    default:
      hipLaunchKernelGGL(importance_kernel<8>, grid, dim3(kBlock), 0, st, c->hi_acc, probs_hi, c->n_hi, c->cap_hi,
                         c->q_heads, c->kv_heads);
  }
  return check_launch("mikv_importance_update");
}

extern "C" size_t mikv_resident_bytes(void) { return (size_t)mikv::resident_budget(); }

extern "C" int mikv_set_resident_bytes(size_t bytes) {
  if (bytes > ((size_t)1 << 62)) return mikv::set_error(MIKV_ERR_INVALID_ARG, "mikv_set_resident_bytes: %zu bytes is out of range", bytes);
  mikv::g_resident_bytes.store((int64_t)bytes, std::memory_order_relaxed);
  return MIKV_OK;
}
