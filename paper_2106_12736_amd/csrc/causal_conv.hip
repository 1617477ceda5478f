// Causal convolution of each channel with its own short kernel, and its backward.
//
//   p[t][d] = bias[d] + sum_j w[d][j] x[t - n + 1 + j][d],  y = p or silu(p)
//   gp = gy silu'(p);  gx[t] = sum_j w[j] gp[t + n - 1 - j];  gw[j] = sum_t gp[t] x[t - n + 1 + j]
//
// A thread owns V adjacent channels of a run of tokens and walks along it with the last n - 1
// rows in registers, so each input crosses HBM once but for the n - 1 rows in front of a run.
// Both directions are bound by HBM: no channel shares anything with another, and a token
// takes n multiply-adds a channel.  8 x 2048 tokens, 4096 channels, 4 taps, bf16: forward 65 to 68 us (4.1 TB/s),
// backward 107 to 114 us (3.8 to 3.5 TB/s), in float32 4.7 and 4.5 TB/s; a large copy runs at 5.1.
#include "sequence.h"

namespace fdc {

struct ConvGrid {
  int CV;     // groups of V channels
  int run;    // tokens a thread walks
  int tiles;  // runs a sequence
};

template <class T, int V>
__device__ __forceinline__ Pack<T, V> row_or_zero(const T *base, int64_t stride, int t, bool live, int nch) {
  return live ? load_some<T, V>(base + (int64_t)t * stride, nch) : Pack<T, V>{};
}
template <class T, int V>
__device__ __forceinline__ void unpack(float (&f)[V], const Pack<T, V> &x) {
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = x.at(i);
}

// Token t of a sequence and, before it, of its state: zero before both and from `len` on.
template <class T, int V>
__device__ __forceinline__ Pack<T, V> token_row(const T *xb, int64_t stride, const T *state, int D, int n, int t,
                                                int len, int nch) {
  return t >= 0 ? row_or_zero<T, V>(xb, stride, t, t < len, nch)
                : row_or_zero<T, V>(state, D, t + n - 1, state != nullptr, nch);
}

// The taps [V][N] and biases of a thread's channels (those of channels that are not there are 0): rows of w
// lie one after another, so they are read in pieces of four whatever N is.
template <int V, int N>
__device__ __forceinline__ void load_taps(float (&w)[N][V], float (&bias)[V], const float *wp, const float *bp, int c0,
                                          int nch) {
  static_assert(V * N % 4 == 0);
#pragma unroll
  for (int m = 0; m < V * N / 4; ++m) {
    const int n = nch * N - 4 * m;
    const Pack<float, 4> x = n > 0 ? load_some<float, 4>(wp + (int64_t)c0 * N + 4 * m, n) : Pack<float, 4>{};
#pragma unroll
    for (int e = 0; e < 4; ++e) w[(4 * m + e) % N][(4 * m + e) / N] = x.at(e);
  }
  const Pack<float, V> x = bp ? load_some<float, V>(bp + c0, nch) : Pack<float, V>{};
#pragma unroll
  for (int i = 0; i < V; ++i) bias[i] = x.at(i);
}

constexpr int kConvUnroll = 4;  // tokens loaded together, while the four before them are worked on

template <class T, int V, int N>
__global__ __launch_bounds__(256) void k_causal_conv_fwd(fdc_causal_conv_args a, ConvGrid cg) {
  const unsigned id = blockIdx.x * 256u + threadIdx.x;
  const int tile = id / cg.CV, c0 = (id - tile * cg.CV) * V, b = blockIdx.y;
  if (tile >= cg.tiles) return;
  const int nch = min(V, a.D - c0), len = length_of(a.lengths, b, a.L);
  const T *xb = static_cast<const T *>(a.x.p) + b * a.x.batch_stride + c0;
  T *yb = static_cast<T *>(a.y.p) + b * a.y.batch_stride + c0;
  const T *st = a.state ? static_cast<const T *>(a.state) + ((int64_t)b * (N - 1)) * a.D + c0 : nullptr;
  const int t0 = tile * cg.run, t1 = min(a.L, t0 + cg.run);

  float w[N][V], bias[V], x[N - 1 + kConvUnroll][V];
  load_taps<V, N>(w, bias, a.w, a.bias, c0, nch);
#pragma unroll
  for (int k = 0; k < N - 1; ++k)
    unpack(x[k], token_row<T, V>(xb, a.x.token_stride, st, a.D, N, t0 - (N - 1) + k, len, nch));
  Pack<T, V> next[kConvUnroll];
  const int end = min(len, t1);
  auto fetch = [&](int t) {
#pragma unroll
    for (int u = 0; u < kConvUnroll; ++u) next[u] = row_or_zero<T, V>(xb, a.x.token_stride, t + u, t + u < end, nch);
  };
  fetch(t0);
  if (tile == 0 && a.new_state != nullptr) {
    // rows len - (n - 1) .. len - 1 of the sequence with its state in front; only this thread reads
    // these channels' state (a run is no shorter than n - 1), and all of it is read before
    // new_state, which may be the same memory, is written
    Pack<T, V> keep[N];
#pragma unroll
    for (int k = 0; k < N - 1; ++k)
      keep[k] = token_row<T, V>(xb, a.x.token_stride, st, a.D, N, len - (N - 1) + k, len, nch);
    T *ns = static_cast<T *>(a.new_state) + ((int64_t)b * (N - 1)) * a.D + c0;
#pragma unroll
    for (int k = 0; k < N - 1; ++k) {
      float f[V];
      unpack(f, keep[k]);
      store_some<T, V>(ns + (int64_t)k * a.D, f, nch);
    }
  }
  for (int t = t0; t < t1; t += kConvUnroll) {
#pragma unroll
    for (int u = 0; u < kConvUnroll; ++u) unpack(x[N - 1 + u], next[u]);
    if (t + kConvUnroll < t1) fetch(t + kConvUnroll);
#pragma unroll
    for (int u = 0; u < kConvUnroll; ++u) {
      float y[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float p = bias[i];
#pragma unroll
        for (int j = 0; j < N; ++j) p = fmaf(w[j][i], x[u + j][i], p);
        y[i] = t + u < len ? (a.silu ? p * sigmoid(p) : p) : 0.f;
      }
      if (t + u < t1) store_some<T, V>(yb + (int64_t)(t + u) * a.y.token_stride, y, nch);
    }
#pragma unroll
    for (int k = 0; k < N - 1; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) x[k][i] = x[k + kConvUnroll][i];
  }
}

// gx of the run's tokens needs gp of n - 1 tokens past it, which are formed here too (their part
// of gw belongs to the next run).  part [B * tiles][n + 1][D]: the run's sums for gw and gbias.
template <class T, int V, int N>
__global__ __launch_bounds__(256) void k_causal_conv_bwd(fdc_causal_conv_args a, fdc_tokens gy, fdc_tokens gx,
                                                         float *__restrict__ part, ConvGrid cg) {
  const unsigned id = blockIdx.x * 256u + threadIdx.x;
  const int tile = id / cg.CV, c0 = (id - tile * cg.CV) * V, b = blockIdx.y;
  if (tile >= cg.tiles) return;
  const int nch = min(V, a.D - c0), len = length_of(a.lengths, b, a.L);
  const T *xb = static_cast<const T *>(a.x.p) + b * a.x.batch_stride + c0;
  const T *gyb = static_cast<const T *>(gy.p) + b * gy.batch_stride + c0;
  T *gxb = gx.p ? static_cast<T *>(gx.p) + b * gx.batch_stride + c0 : nullptr;
  const T *st = a.state ? static_cast<const T *>(a.state) + ((int64_t)b * (N - 1)) * a.D + c0 : nullptr;
  const int t0 = tile * cg.run, t1 = min(a.L, t0 + cg.run);

  float w[N][V], bias[V], x[N - 1 + kConvUnroll][V], gp[N - 1 + kConvUnroll][V], gw[N][V], gb[V];
  load_taps<V, N>(w, bias, a.w, a.bias, c0, nch);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    gb[i] = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) gw[j][i] = 0.f;
  }
#pragma unroll
  for (int k = 0; k < N - 1; ++k) {
    unpack(x[k], token_row<T, V>(xb, a.x.token_stride, st, a.D, N, t0 - (N - 1) + k, len, nch));
#pragma unroll
    for (int i = 0; i < V; ++i) gp[k][i] = 0.f;
  }
  const int last = gxb ? t1 + N - 1 : t1;  // gp is wanted for t < last
  const int end = min(len, last), own = min(len, t1);  // tokens loaded; tokens of this run's sums
  Pack<T, V> next_x[kConvUnroll], next_g[kConvUnroll];
  auto fetch = [&](int t) {
#pragma unroll
    for (int u = 0; u < kConvUnroll; ++u) {
      next_x[u] = row_or_zero<T, V>(xb, a.x.token_stride, t + u, t + u < end, nch);
      next_g[u] = row_or_zero<T, V>(gyb, gy.token_stride, t + u, t + u < end, nch);
    }
  };
  fetch(t0);
  for (int t = t0; t < last; t += kConvUnroll) {
    float g[kConvUnroll][V];
#pragma unroll
    for (int u = 0; u < kConvUnroll; ++u) {
      unpack(x[N - 1 + u], next_x[u]);
      unpack(g[u], next_g[u]);
    }
    if (t + kConvUnroll < last) fetch(t + kConvUnroll);
#pragma unroll
    for (int u = 0; u < kConvUnroll; ++u) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float v = g[u][i];
        if (a.silu) {
          float p = bias[i];
#pragma unroll
          for (int j = 0; j < N; ++j) p = fmaf(w[j][i], x[u + j][i], p);
          const float sg = sigmoid(p);
          v *= sg * (1.f + p * (1.f - sg));
        }
        gp[N - 1 + u][i] = t + u < len ? v : 0.f;
      }
      // (a product with 0 would not do: a row of the window may hold what is not finite)
      if (t + u < own) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float v = gp[N - 1 + u][i];
          gb[i] += v;
#pragma unroll
          for (int j = 0; j < N; ++j) gw[j][i] = fmaf(v, x[u + j][i], gw[j][i]);
        }
      }
      const int to = t + u - (N - 1);  // gp[to .. t + u] are here
      if (gxb && to >= t0 && to < t1) {
        float o[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          float s = 0.f;
#pragma unroll
          for (int j = 0; j < N; ++j) s = fmaf(w[j][i], gp[u + N - 1 - j][i], s);
          o[i] = to < len ? s : 0.f;
        }
        store_some<T, V>(gxb + (int64_t)to * gx.token_stride, o, nch);
      }
    }
#pragma unroll
    for (int k = 0; k < N - 1; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        x[k][i] = x[k + kConvUnroll][i];
        gp[k][i] = gp[k + kConvUnroll][i];
      }
  }
  if (part != nullptr) {
    float *pr = part + ((int64_t)b * cg.tiles + tile) * (N + 1) * a.D + c0;
#pragma unroll
    for (int j = 0; j < N; ++j) store_some<float, V>(pr + (int64_t)j * a.D, gw[j], nch);
    store_some<float, V>(pr + (int64_t)N * a.D, gb, nch);
  }
}

namespace {

// Runs as long as leave at least `want` threads (so that the rows in front of a run are few), in powers of
// two from 8 (no shorter than the n - 1 <= 7 tokens of a state) to `most`.  (The case above: runs of 8 163
// us forward and 198 backward, of 64 63 and 116, of 128 82 and 94, of 256 147 and 138; a sequence of
// 4096 tokens of 2048 channels: runs of 16 15 and 19, of 64 23 and 37.)
ConvGrid conv_grid(int B, int L, int D, int V, int most, long long want) {
  ConvGrid cg;
  cg.CV = (int)ceil_div(D, V);
  cg.run = 8;
  while (cg.run < most && (long long)B * cg.CV * ceil_div(L, 2 * cg.run) >= want) cg.run *= 2;
  cg.tiles = (int)ceil_div(L, cg.run);
  return cg;
}

template <class T>
constexpr int kFwdV = sizeof(T) == 2 ? 8 : 4;  // 16 bytes a lane
constexpr int kBwdV = 4;  // two windows and the sums of gw in registers

ConvGrid bwd_grid(int B, int L, int D) { return conv_grid(B, L, D, kBwdV, 128, 1 << 17); }

template <class F>
hipError_t by_taps(int n, F &&f) {
  switch (n) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 3: return f(std::integral_constant<int, 3>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 5: return f(std::integral_constant<int, 5>{});
    case 6: return f(std::integral_constant<int, 6>{});
    case 7: return f(std::integral_constant<int, 7>{});
    default: return f(std::integral_constant<int, 8>{});
  }
}

}  // namespace

hipError_t launch_causal_conv_fwd(const fdc_causal_conv_args &a, hipStream_t s) {
  return by_dtype(a.dtype, [&](auto tag) {
    using T = decltype(tag);
    constexpr int V = kFwdV<T>;
    return by_taps(a.n, [&](auto taps) {
      const ConvGrid cg = conv_grid(a.B, a.L, a.D, V, 64, 1 << 17);
      const long long blocks = ceil_div((long long)cg.CV * cg.tiles, 256);
      return timed_launch("causal_conv_fwd", k_causal_conv_fwd<T, V, taps.value>, dim3((unsigned)blocks, a.B),
                          dim3(256), 0, s, a, cg);
    });
  });
}

size_t causal_conv_bwd_ws(int dtype, int B, int L, int D, int n) {
  return (size_t)B * bwd_grid(B, L, D).tiles * (n + 1) * D * sizeof(float);
}

hipError_t launch_causal_conv_bwd(const fdc_causal_conv_args &a, const fdc_tokens &gy, const fdc_tokens &gx, float *gw,
                                  float *gbias, float *part, hipStream_t s) {
  const ConvGrid cg = bwd_grid(a.B, a.L, a.D);
  float *p = gw || gbias ? part : nullptr;
  hipError_t e = by_dtype(a.dtype, [&](auto tag) {
    using T = decltype(tag);
    return by_taps(a.n, [&](auto taps) {
      const long long blocks = ceil_div((long long)cg.CV * cg.tiles, 256);
      return timed_launch("causal_conv_bwd", k_causal_conv_bwd<T, kBwdV, taps.value>, dim3((unsigned)blocks, a.B),
                          dim3(256), 0, s, a, gy, gx, p, cg);
    });
  });
  if (e != hipSuccess || p == nullptr) return e;
  ColSegments segs{};
  segs.count = 2;
  segs.seg[0] = ColSegment{gw, a.n * a.D, a.D, a.n};
  segs.seg[1] = ColSegment{gbias, a.D, a.D, 1};
  return launch_col_sums(p, (long long)a.B * cg.tiles, (long long)(a.n + 1) * a.D, segs, s);
}

}  // namespace fdc
