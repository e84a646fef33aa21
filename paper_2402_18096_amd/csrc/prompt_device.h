// Device pieces shared by the kernels over whole prompts (prefill.hip,
// prompt.hip): 32x32x16 fp16 MFMA tiles whose streamed rows pass through LDS.
#ifndef MIKV_PROMPT_DEVICE_H
#define MIKV_PROMPT_DEVICE_H

#include "mikv_internal.h"

namespace mikv {

namespace {

constexpr int kThreads = 256;
constexpr int kWaveRows = 64;          // stationary rows per wave (two 32-row tiles)
constexpr int kRowWords = kHeadDim / 8;  // 16-byte words per fp16 row
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.69314718055994531f;

typedef _Float16 h8_t __attribute__((ext_vector_type(8)));
typedef float f16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u4_t __attribute__((ext_vector_type(4)));

__device__ inline h8_t as_h8(u4_t v) { return __builtin_bit_cast(h8_t, v); }

// Rows of an LDS tile: 16-byte word c of row r sits at word c ^ (r % 16), so
// that the 16 lanes that one LDS cycle serves touch every bank once, both
// when a row is written and when 16 rows are read at the same word.
__device__ inline int lds_word(int row, int c) { return row * kRowWords + (c ^ (row & 15)); }

// Byte offset of the lane's word 0 of row 0 of a tile; its word i of row r
// (r a multiple of 32) is at (offset ^ 32 i) + 256 r.
__device__ inline uint32_t tile_offset() {
  const int lane = threadIdx.x & 63;
  return 16u * (uint32_t)lds_word(lane & 31, lane >> 5);
}
__device__ inline u4_t read_word(const u4_t *lds, uint32_t off, int row0, int i) {
  return *reinterpret_cast<const u4_t *>(reinterpret_cast<const char *>(lds) + (off ^ (32u * i)) + 256 * row0);
}
__device__ inline void read_tile(const u4_t *lds, uint32_t off, int row0, u4_t op[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) op[i] = read_word(lds, off, row0, i);
}

__device__ inline void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }  // vmcnt(0)

__device__ inline f16_t splat(float v) {
  f16_t d;
#pragma unroll
  for (int r = 0; r < 16; ++r) d[r] = v;
  return d;
}

// 32 x 32 logits: rows `key` tile, columns `query` tile.
__device__ inline f16_t logits(const u4_t key[8], const u4_t query[8]) {
  f16_t d = splat(0.0f);
#pragma unroll
  for (int i = 0; i < 8; ++i) d = __builtin_amdgcn_mfma_f32_32x32x16_f16(as_h8(key[i]), as_h8(query[i]), d, 0, 0, 0);
  return d;
}

__device__ inline int tile_row(int r) { return 8 * (r >> 2) + 4 * ((threadIdx.x & 63) >> 5) + (r & 3); }

// Block -> (unit, index) with index 0 the longest.  A unit's blocks stream the
// same head's rows.  Workgroups go to the eight XCDs in turn: a unit keeps to
// one XCD, and `run` of its blocks, about equally long, follow each other there,
// so that its L2 serves most of their rows; over the runs the longest go first
// for every unit, so that the grid ends on its shortest blocks.  False: no work
// (the last group's units count as eight, the last run's blocks as `run`).
__device__ inline bool block_unit(int units, int per_unit, int run, int &unit, int &idx) {
  const int groups = (units + 7) / 8, e = blockIdx.x >> 3;
  const int r = e / (groups * run), rem = e % (groups * run);
  unit = 8 * (rem / run) + (blockIdx.x & 7);
  idx = r * run + rem % run;
  return unit < units && idx < per_unit;
}

}  // namespace

}  // namespace mikv

#endif  // MIKV_PROMPT_DEVICE_H
