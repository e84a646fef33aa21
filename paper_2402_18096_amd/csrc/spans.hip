// The keys that each query of a prompt sees, as one interval [begin, end) per
// query: documents (runs of equal ids), a prefix seen from everywhere in its
// document, a sliding window and padding all come down to it, so the attention
// kernels know one mask.
// Bound: latency (the ids are read twice, the interval is written once).  One
// block per sequence; thread t owns the t-th stretch of tokens, finds the first
// and last document border in it, and two scans over the threads give every
// stretch the border before it and the one after it.
#include "../../include/mikv_layer.h"
#include "mikv_internal.h"

namespace mikv {

namespace {

constexpr int kSpanBlock = 1024, kSpanWaves = kSpanBlock / 64;

__global__ __launch_bounds__(kSpanBlock) void mask_spans_kernel(const int32_t *documents, const int32_t *prefix, int T,
                                                               int window, int32_t *begin, int32_t *end) {
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t *ids = documents ? documents + (int64_t)b * T : nullptr;
  const int per = (T + kSpanBlock - 1) / kSpanBlock;
  const int t0 = (int)min((int64_t)tid * per, (int64_t)T), t1 = min(t0 + per, T);
  auto border = [&](int i) { return ids[i] != ids[i - 1]; };  // i >= 1
  int first = T, last = 0;  // borders inside the stretch: the first, and the last
  if (ids) {
    for (int i = max(t0, 1); i < t1; ++i)
      if (border(i)) {
        first = min(first, i);
        last = i;
      }
  }
  // before: the largest `last` of the threads before this one; after: the
  // smallest `first` of those behind it
  int before = last, after = first;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(before, o, 64), y = __shfl_down(after, o, 64);
    if (lane >= o) before = max(before, x);
    if (lane + o < 64) after = min(after, y);
  }
  __shared__ int s_last[kSpanWaves], s_first[kSpanWaves];
  if (lane == 63) s_last[wave] = before;
  if (lane == 0) s_first[wave] = after;
  __syncthreads();
  const int up = __shfl_up(before, 1, 64), down = __shfl_down(after, 1, 64);
  before = lane == 0 ? 0 : up;
  after = lane == 63 ? T : down;
  for (int w = 0; w < wave; ++w) before = max(before, s_last[w]);
  for (int w = wave + 1; w < kSpanWaves; ++w) after = min(after, s_first[w]);
  const int pre = prefix ? prefix[b] : 0;
  int start = before, stop = -1;  // the run of token i is [start, stop)
  for (int i = t0; i < t1; ++i) {
    if (ids && i > 0 && border(i)) {
      start = i;
      stop = -1;
    }
    if (stop < 0) {
      stop = after;
      if (ids)
        for (int j = i + 1; j < t1; ++j)
          if (border(j)) {
            stop = j;
            break;
          }
    }
    int lo = start, hi = max(i + 1, min(stop, pre));
    if (window > 0) lo = max(lo, i + 1 - min(window, i + 1));
    if (ids && ids[i] < 0) lo = hi = 0;
    begin[(int64_t)b * T + i] = lo;
    end[(int64_t)b * T + i] = hi;
  }
}

}  // namespace

}  // namespace mikv

using namespace mikv;

extern "C" int mikv_mask_spans(const int32_t *documents, const int32_t *prefix, int32_t batch, int32_t tokens,
                               int32_t window, int32_t *begin, int32_t *end, void *stream) {
  if (!begin || !end) return set_error(MIKV_ERR_INVALID_ARG, "mikv_mask_spans: NULL output");
  if (batch < 1 || tokens < 1 || window < 0)
    return set_error(MIKV_ERR_INVALID_ARG, "mikv_mask_spans: batch and tokens >= 1, window >= 0 expected");
  if (tokens > 1 << 30) return set_error(MIKV_ERR_UNSUPPORTED, "mikv_mask_spans: over 2^30 tokens");
  if (((uintptr_t)documents | (uintptr_t)prefix | (uintptr_t)begin | (uintptr_t)end) % 4)
    return set_error(MIKV_ERR_INVALID_ARG, "mikv_mask_spans: misaligned pointer");
  hipLaunchKernelGGL(mask_spans_kernel, dim3(batch), dim3(kSpanBlock), 0, (hipStream_t)stream, documents, prefix, tokens,
                     window, begin, end);
  return check_launch("mikv_mask_spans");
}
