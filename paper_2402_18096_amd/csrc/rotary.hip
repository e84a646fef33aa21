// Rotary positions: the rows of a layer's projection (queries, keys, values)
// to rotated fp16 rows in the layout that the prompt's calls and the cache
// take, in one launch:
//   (a, b) -> m (a cos t - b sin t, b cos t + a sin t),  t = 2 pi pos w_p.
// The phase pos * w_p is taken modulo one turn in 64-bit fixed point (w_p in
// units of 2^-64 turns), so it is as exact at position 10^6 as at 1 and needs no
// table of angles; sine and cosine are those of half turns, whose argument
// reduction is exact.
// Bound: reading and writing every row once.  A thread takes 2 W channels (W
// pairs) of one token and turns them in `hp` heads, one after the other, so the
// sines cost a fraction of the loads; eight threads of W = 8 cover a row in
// 16-byte words.
#include <algorithm>
#include <cmath>

#include "../../include/mikv_layer.h"
#include "mikv_internal.h"

namespace mikv {

namespace {

struct RotTensor {
  const void *x;
  void *y;
  int64_t xb, xh, xt, yb, yh, yt;  // strides in elements
  int heads, rotate;
};

struct RotArgs {
  RotTensor t[3];
  int n, heads, hp;  // heads over all tensors; heads per thread
  int rows, tokens;  // rows = batch * tokens
  const int32_t *positions;
  int pos0;
  const uint64_t *freq;
  int half;  // rot_dim / 2
  float magnitude;
};

template <int TYPE>
struct Elem;
template <>
struct Elem<MIKV_F16> {
  typedef _Float16 type;
};
template <>
struct Elem<MIKV_BF16> {
  typedef __bf16 type;
};
template <>
struct Elem<MIKV_F32> {
  typedef float type;
};

// N elements at p, in words of at most 16 bytes (p aligned to min(16, N elements)).
template <class T, int N>
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Pack {
  T v[N];
};

template <class T, int N>
__device__ inline void load(const T *p, float x[N]) {
  const Pack<T, N> w = *reinterpret_cast<const Pack<T, N> *>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = (float)w.v[i];
}

template <class T, int N>
__device__ inline void store(T *p, const float x[N]) {
  Pack<T, N> w;
#pragma unroll
  for (int i = 0; i < N; ++i) w.v[i] = (T)x[i];
  *reinterpret_cast<Pack<T, N> *>(p) = w;
}

template <int X, int Y, int W, bool IL>
__global__ __launch_bounds__(256) void rotary_kernel(RotArgs A) {
  typedef typename Elem<X>::type TX;
  typedef typename Elem<Y>::type TY;
  constexpr int S = kHeadDim / (2 * W);  // threads of a row
  const int id = blockIdx.x * blockDim.x + threadIdx.x;
  const int row = id / S, c = id % S;
  if (row >= A.rows) return;
  const int b = row / A.tokens, t = row % A.tokens;
  // channels [c0, c0 + W) and [c1, c1 + W): both halves' of W pairs, or W pairs of
  // neighbours, or 2 W channels past the rotated ones (W divides half)
  const bool turned = W * c < A.half;
  const int c0 = IL || !turned ? 2 * W * c : W * c;
  const int c1 = IL || !turned ? c0 + W : c0 + A.half;
  float cs[W], sn[W];
  if (turned) {
    const int64_t pos = A.positions ? A.positions[row] : (int64_t)A.pos0 + t;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const int32_t phase = (int32_t)((uint64_t)pos * A.freq[W * c + i] >> 32);
      sincospif((float)phase * 0x1p-31f, &sn[i], &cs[i]);
      sn[i] *= A.magnitude;
      cs[i] *= A.magnitude;
    }
  }
  const int h0 = blockIdx.y * A.hp, h1 = min(h0 + A.hp, A.heads);
  for (int h = h0; h < h1; ++h) {  // wave-uniform
    int k = 0, hh = h;
    while (hh >= A.t[k].heads) hh -= A.t[k++].heads;
    const RotTensor &R = A.t[k];
    const TX *x = (const TX *)R.x + b * R.xb + hh * R.xh + t * R.xt;
    TY *y = (TY *)R.y + b * R.yb + hh * R.yh + t * R.yt;
    float u[W], v[W], p[W], q[W];
    load<TX, W>(x + c0, u);
    load<TX, W>(x + c1, v);
    if (turned && R.rotate) {
      if constexpr (IL) {
        float z[2 * W];
#pragma unroll
        for (int i = 0; i < W; ++i) {
          z[i] = u[i];
          z[W + i] = v[i];
        }
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const float a = z[2 * i], e = z[2 * i + 1];
          z[2 * i] = a * cs[i] - e * sn[i];
          z[2 * i + 1] = e * cs[i] + a * sn[i];
        }
#pragma unroll
        for (int i = 0; i < W; ++i) {
          p[i] = z[i];
          q[i] = z[W + i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < W; ++i) {
          p[i] = u[i] * cs[i] - v[i] * sn[i];
          q[i] = v[i] * cs[i] + u[i] * sn[i];
        }
      }
      store<TY, W>(y + c0, p);
      store<TY, W>(y + c1, q);
    } else {
      store<TY, W>(y + c0, u);
      store<TY, W>(y + c1, v);
    }
  }
}

template <int X, int Y, int W>
void launch_rotary(const RotArgs &A, bool interleaved, hipStream_t st) {
  const int64_t threads = (int64_t)A.rows * (kHeadDim / (2 * W));
  const int block = threads <= 4096 ? 64 : 256;  // a few tokens: more blocks, one wave each
  const dim3 grid((unsigned)((threads + block - 1) / block), (A.heads + A.hp - 1) / A.hp);
  if (interleaved)
    hipLaunchKernelGGL((rotary_kernel<X, Y, W, true>), grid, dim3(block), 0, st, A);
  else
    hipLaunchKernelGGL((rotary_kernel<X, Y, W, false>), grid, dim3(block), 0, st, A);
}

template <int X, int Y>
void launch_rotary_w(const RotArgs &A, int w, bool interleaved, hipStream_t st) {
  if (w == 8)
    launch_rotary<X, Y, 8>(A, interleaved, st);
  else if (w == 2)
    launch_rotary<X, Y, 2>(A, interleaved, st);
  else
    launch_rotary<X, Y, 1>(A, interleaved, st);
}

}  // namespace

}  // namespace mikv

using namespace mikv;

extern "C" int mikv_rotary_frequencies(const mikv_rotary_scheme *s, uint64_t *freq, float *magnitude) {
  const char *who = "mikv_rotary_frequencies";
  if (!s || !freq || !magnitude) return set_error(MIKV_ERR_INVALID_ARG, "%s: NULL pointer", who);
  if (s->rot_dim < 2 || s->rot_dim > kHeadDim || s->rot_dim % 2)
    return set_error(MIKV_ERR_INVALID_ARG, "%s: rot_dim must be even, 2 .. %d (got %d)", who, kHeadDim, s->rot_dim);
  if (s->scaling < MIKV_ROTARY_PLAIN || s->scaling > MIKV_ROTARY_YARN)
    return set_error(MIKV_ERR_INVALID_ARG, "%s: unknown scaling %d", who, s->scaling);
  if (!(s->base > 1.0) || !std::isfinite(s->base)) return set_error(MIKV_ERR_INVALID_ARG, "%s: base must be > 1", who);
  const bool scaled = s->scaling != MIKV_ROTARY_PLAIN;
  const bool blended = s->scaling == MIKV_ROTARY_BANDS || s->scaling == MIKV_ROTARY_YARN;
  if (scaled && (!(s->factor >= 1.0) || !std::isfinite(s->factor)))
    return set_error(MIKV_ERR_INVALID_ARG, "%s: factor must be >= 1", who);
  if (blended && (!(s->original_length > 0.0) || !std::isfinite(s->original_length) || !(s->low > 0.0) ||
                  !(s->high > s->low) || !std::isfinite(s->high)))
    return set_error(MIKV_ERR_INVALID_ARG, "%s: original_length > 0 and 0 < low < high expected", who);
  if (s->scaling == MIKV_ROTARY_NTK && s->rot_dim == 2)
    return set_error(MIKV_ERR_INVALID_ARG, "%s: NTK scaling needs rot_dim > 2", who);
  const long double r = s->rot_dim, two_pi = 2.0L * acosl(-1.0L), f = scaled ? s->factor : 1.0L;
  long double base = s->base;
  if (s->scaling == MIKV_ROTARY_NTK) base *= powl(f, r / (r - 2.0L));
  auto pair_of = [&](long double turns) { return r * logl((long double)s->original_length / (turns * two_pi)) / (2.0L * logl(base)); };
  for (int p = 0; p < s->rot_dim / 2; ++p) {
    long double w = powl(base, -2.0L * p / r);
    if (s->scaling == MIKV_ROTARY_LINEAR) w /= f;
    if (blended) {
      long double keep;
      if (s->scaling == MIKV_ROTARY_BANDS) {
        keep = (s->original_length * w / two_pi - s->low) / ((long double)s->high - s->low);
      } else {
        const long double first = std::max(0.0L, floorl(pair_of(s->high))), last = std::min(r - 1.0L, ceill(pair_of(s->low)));
        keep = 1.0L - ((long double)p - first) / std::max(last - first, 0.001L);
      }
      keep = std::min(1.0L, std::max(0.0L, keep));
      w = w * keep + w / f * (1.0L - keep);
    }
    freq[p] = (uint64_t)llroundl(ldexpl(w / two_pi, 62)) << 2;  // below one sixth of a turn
  }
  *magnitude = s->scaling == MIKV_ROTARY_YARN ? (float)(0.1L * logl(f) + 1.0L) : 1.0f;
  return MIKV_OK;
}

extern "C" int mikv_rotary(const mikv_heads *tensors, int32_t n, int32_t batch, int32_t tokens, int32_t head_dim,
                           int32_t x_type, int32_t y_type, const int32_t *positions, int32_t pos0, const uint64_t *freq,
                           int32_t rot_dim, int32_t interleaved, float magnitude, void *stream) {
  if (!tensors || !freq) return set_error(MIKV_ERR_INVALID_ARG, "mikv_rotary: NULL pointer");
  if (n < 1 || n > 3 || batch < 1 || tokens < 1)
    return set_error(MIKV_ERR_INVALID_ARG, "mikv_rotary: 1 to 3 tensors, batch and tokens >= 1 expected");
  if (head_dim != kHeadDim) return set_error(MIKV_ERR_UNSUPPORTED, "mikv_rotary: head_dim must be %d", kHeadDim);
  if (rot_dim < 2 || rot_dim > kHeadDim || rot_dim % 2)
    return set_error(MIKV_ERR_INVALID_ARG, "mikv_rotary: rot_dim must be even, 2 .. %d (got %d)", kHeadDim, rot_dim);
  if (x_type < MIKV_F16 || x_type > MIKV_F32 || (y_type != x_type && y_type != MIKV_F16))
    return set_error(MIKV_ERR_INVALID_ARG, "mikv_rotary: y_type must be x_type or MIKV_F16 (got %d -> %d)", x_type, y_type);
  if ((int64_t)batch * tokens > 1 << 24) return set_error(MIKV_ERR_UNSUPPORTED, "mikv_rotary: over 2^24 tokens");
  if ((uintptr_t)positions % 4 || (uintptr_t)freq % 8)
    return set_error(MIKV_ERR_INVALID_ARG, "mikv_rotary: positions or freq misaligned");
  const int xs = x_type == MIKV_F32 ? 4 : 2, ys = y_type == MIKV_F32 ? 4 : 2;
  RotArgs A{};
  // bytes of alignment that every row has
  uint64_t any_x = 0, any_y = 0;
  int64_t heads = 0;
  for (int i = 0; i < n; ++i) {
    const mikv_heads &h = tensors[i];
    if (!h.x || !h.y) return set_error(MIKV_ERR_INVALID_ARG, "mikv_rotary: NULL tensor");
    if (h.heads < 1) return set_error(MIKV_ERR_INVALID_ARG, "mikv_rotary: heads must be >= 1");
    if (h.x == h.y && x_type != y_type)
      return set_error(MIKV_ERR_INVALID_ARG, "mikv_rotary: in place needs one type");
    RotTensor &R = A.t[i];
    R.x = h.x;
    R.y = h.y;
    R.xb = h.x_stride[0], R.xh = h.x_stride[1], R.xt = h.x_stride[2];
    R.yb = h.y_stride[0], R.yh = h.y_stride[1], R.yt = h.y_stride[2];
    if (h.x == h.y && ((batch > 1 && R.xb != R.yb) || (h.heads > 1 && R.xh != R.yh) || (tokens > 1 && R.xt != R.yt)))
      return set_error(MIKV_ERR_INVALID_ARG, "mikv_rotary: in place needs the same strides");
    if ((batch > 1 && !R.yb) || (h.heads > 1 && !R.yh) || (tokens > 1 && !R.yt))
      return set_error(MIKV_ERR_INVALID_ARG, "mikv_rotary: the output's rows share memory (stride 0)");
    R.heads = h.heads;
    R.rotate = h.rotate;
    heads += h.heads;
    any_x |= (uint64_t)(uintptr_t)h.x | (uint64_t)((R.xb | R.xh | R.xt) * xs);
    any_y |= (uint64_t)(uintptr_t)h.y | (uint64_t)((R.yb | R.yh | R.yt) * ys);
  }
  if (any_x % xs || any_y % ys) return set_error(MIKV_ERR_INVALID_ARG, "mikv_rotary: x or y not aligned to its type");
  if (heads > 65536) return set_error(MIKV_ERR_UNSUPPORTED, "mikv_rotary: over 2^16 heads");
  A.n = n;
  A.heads = (int)heads;
  A.rows = batch * tokens;
  A.tokens = tokens;
  A.positions = positions;
  A.pos0 = pos0;
  A.freq = freq;
  A.half = rot_dim / 2;
  A.magnitude = magnitude;
  // the widest W pairs a thread can take: W divides the pairs, and its words are aligned
  const int w = rot_dim % 16 == 0 && any_x % 16 == 0 && any_y % 16 == 0                ? 8
                : rot_dim % 4 == 0 && any_x % (2 * xs) == 0 && any_y % (2 * ys) == 0 ? 2
                                                                                       : 1;
  // Heads per thread: eight share the sines of a thread once there are threads
  // enough for the chip without them; a few tokens take a thread per head.
  const int64_t all = (int64_t)A.rows * (kHeadDim / (2 * w)) * heads;
  A.hp = (int)std::min<int64_t>(8, std::max<int64_t>({1, all >> 18, (heads + 65534) / 65535}));
  hipStream_t st = (hipStream_t)stream;
  const bool il = interleaved != 0;
  if (x_type == MIKV_F16)
    launch_rotary_w<MIKV_F16, MIKV_F16>(A, w, il, st);
  else if (x_type == MIKV_BF16 && y_type == MIKV_BF16)
    launch_rotary_w<MIKV_BF16, MIKV_BF16>(A, w, il, st);
  else if (x_type == MIKV_BF16)
    launch_rotary_w<MIKV_BF16, MIKV_F16>(A, w, il, st);
  else if (y_type == MIKV_F32)
    launch_rotary_w<MIKV_F32, MIKV_F32>(A, w, il, st);
  else
    launch_rotary_w<MIKV_F32, MIKV_F16>(A, w, il, st);
  return check_launch("mikv_rotary");
}
