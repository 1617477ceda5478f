// Rotary positions of several axes: each pair of channels of every head is turned by position * frequency.
//
//   (u, v) -> (u cos(a) - v sin(a), u sin(a) + v cos(a));   the gradient is the turn by -a.
//
// A pass over x and y (HBM-bound: 32768 tokens of 16 heads of 128 bf16, 268 MB, 64 us, 4.2 TB/s).  The angle of a pair is
// that of every head of the token, so a thread holds the cosines and sines of VP pairs (a 16-byte piece of either half) and
// goes through the heads with them.
#include "launch_limit.h"
#include "sequence.h"

namespace fdc {

constexpr int kRotaryThreads = 256;

// Cosine and sine of pos * freq.  The angle is formed in turns and reduced to an eighth of a turn either way in 64
// bits (a position of 2^20 alone takes 20 of float32's 24), the rest by its Taylor polynomials, whose
// next terms are below 2e-9.
__device__ __forceinline__ void cos_sin(int pos, float freq, float &c, float &s) {
  const double turns = (double)pos * (double)freq * 0.15915494309189533577;
  const double r = turns - rint(turns), q = rint(4.0 * r);
  const float x = (float)(fma(q, -0.25, r) * 6.28318530717958647693);
  const float x2 = x * x;
  const float sx = fmaf(x * x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), x);
  const float cx =
      fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const int k = (int)q & 3;  // quarter turns
  c = k & 1 ? sx : cx;
  s = k & 1 ? cx : sx;
  if (k == 1 || k == 2) c = -c;
  if (k >= 2) s = -s;
}

// Thread (piece, token, run of heads): pieces of VP pairs, then pieces of 2 VP channels that are copied.
template <class T, bool Interleaved>
__global__ __launch_bounds__(kRotaryThreads) void k_rotary(fdc_rotary_args a, int P, int turned, int pieces,
                                                           int runs, int heads, long long total) {
  constexpr int VP = 16 / (int)sizeof(T);
  const long long id = (long long)blockIdx.x * kRotaryThreads + threadIdx.x;
  if (id >= total) return;
  const long long rest = id / pieces;
  const int piece = (int)(id - rest * pieces);
  const long long at = rest / runs;
  const int h0 = (int)(rest - at * runs) * heads, h1 = min(a.H, h0 + heads);
  const int b = (int)(at / a.L), t = (int)(at - (long long)b * a.L);
  const T *x = static_cast<const T *>(a.x.p) + b * a.x.batch_stride + t * a.x.token_stride;
  T *y = static_cast<T *>(a.y.p) + b * a.y.batch_stride + t * a.y.token_stride;
  const bool live = t < length_of(a.lengths, b, a.L);
  if (piece >= turned) {
    const int c = 2 * P + (piece - turned) * 2 * VP;
    for (int h = h0; h < h1; ++h)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int ch = c + half * VP, n = a.D - ch;
        if (n <= 0) break;
        float o[VP] = {};
        if (live) {
          const Pack<T, VP> v = load_some<T, VP>(x + h * a.x.head_stride + ch, n);
#pragma unroll
          for (int i = 0; i < VP; ++i) o[i] = v.at(i);
        }
        store_some<T, VP>(y + h * a.y.head_stride + ch, o, n);
      }
    return;
  }
  const int p0 = piece * VP, n = min(VP, P - p0);
  // the channels of the pairs' first and second members, or the first and second half of the pairs' channels
  const int cu = Interleaved ? 2 * p0 : p0, cv = Interleaved ? 2 * p0 + VP : P + p0;
  const int nu = Interleaved ? min(VP, 2 * n) : n, nv = Interleaved ? 2 * n - VP : n;
  if (!live) {
    const float o[VP] = {};
    for (int h = h0; h < h1; ++h) {
      store_some<T, VP>(y + h * a.y.head_stride + cu, o, nu);
      if (nv > 0) store_some<T, VP>(y + h * a.y.head_stride + cv, o, nv);
    }
    return;
  }
  float c[VP], s[VP];
  const int32_t *pos = a.positions + b * a.pos_batch_stride + t * a.pos_token_stride;
#pragma unroll
  for (int i = 0; i < VP; ++i) {
    const int p = min(p0 + i, P - 1);
    int axis = 0, end = a.pairs[0];
    while (p >= end && axis < a.axes - 1) end += a.pairs[++axis];
    cos_sin(pos[axis], a.freqs[p], c[i], s[i]);
    if (a.inverse) s[i] = -s[i];
  }
  // x and y may be the same memory: a thread reads the channels it writes, before
#pragma unroll 4
  for (int h = h0; h < h1; ++h) {
    const T *xh = x + h * a.x.head_stride;
    T *yh = y + h * a.y.head_stride;
    const Pack<T, VP> u = load_some<T, VP>(xh + cu, nu);
    Pack<T, VP> v{};
    if (nv > 0) v = load_some<T, VP>(xh + cv, nv);
    float ou[VP], ov[VP];
#pragma unroll
    for (int i = 0; i < VP; ++i) {
      if constexpr (Interleaved) {
        // pair i of the piece: elements 2 i and 2 i + 1 of u and v in a row
        const float e = 2 * i < VP ? u.at((2 * i) % VP) : v.at((2 * i) % VP);
        const float f = 2 * i < VP ? u.at((2 * i + 1) % VP) : v.at((2 * i + 1) % VP);
        float(&o)[VP] = 2 * i < VP ? ou : ov;
        o[(2 * i) % VP] = fmaf(e, c[i], -(f * s[i]));
        o[(2 * i + 1) % VP] = fmaf(e, s[i], f * c[i]);
      } else {
        ou[i] = fmaf(u.at(i), c[i], -(v.at(i) * s[i]));
        ov[i] = fmaf(u.at(i), s[i], v.at(i) * c[i]);
      }
    }
    store_some<T, VP>(yh + cu, ou, nu);
    if (nv > 0) store_some<T, VP>(yh + cv, ov, nv);
  }
}

hipError_t launch_rotary(const fdc_rotary_args &a, hipStream_t s) {
  return by_dtype(a.dtype, [&](auto tag) {
    using T = decltype(tag);
    constexpr int VP = 16 / (int)sizeof(T);
    int P = 0;
    for (int i = 0; i < a.axes; ++i) P += a.pairs[i];
    const int turned = (int)ceil_div(P, VP), pieces = turned + (int)ceil_div(a.D - 2 * P, 2 * VP);
    const int heads = rotary_heads((long long)a.B * a.L * pieces, a.H);
    const int runs = (int)ceil_div(a.H, heads);
    const long long total = (long long)a.B * a.L * pieces * runs, blocks = ceil_div(total, kRotaryThreads);
    if (blocks * kRotaryThreads >= (1LL << 32)) return hipErrorInvalidConfiguration;
    return timed_launch("rotary", a.interleaved ? k_rotary<T, true> : k_rotary<T, false>, dim3((unsigned)blocks),
                        dim3(kRotaryThreads), 0, s, a, P, turned, pieces, runs, heads, total);
  });
}

}  // namespace fdc
