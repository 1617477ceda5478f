// The end of a block and the start of the next in one pass over the row: norm of the block's output,
// gate, residual scale and residual, and the norm of the sum.
//
//   fh = f rf, rf = 1 / sqrt(mean(f^2) + eps);  post = fh w_post;  out = x + scale act(gate) post
//   n = out ro w_pre, ro = 1 / sqrt(mean(out^2) + eps)
// Backward, from gout and gn:
//   oh = out ro;  v = gn w_pre;  go = gout + (v - oh mean(v oh)) ro = gx;  gw_pre = sum gn oh
//   gscale = sum go act post;  ggate = go scale post act'(gate);  gpost = go scale act
//   u = gpost w_post;  gf = (u - fh mean(u fh)) rf;  gw_post = sum gpost fh
// The means are of normed rows, of size 1: rf^3 and ro^3 would leave float32's range for rows of 1e13 and
// for rows of zeros under a small eps.
//
// A row is in the registers of the threads that share it, so everything is read and written once;
// both directions are bound by HBM.  Workgroups take row after row and keep the parameters in
// registers (read again for every row they would be more than the row itself), and the next row's
// loads are on their way while a row is worked on.  The sums over a row are formed in float32, across
// the wave by lane moves and across waves through LDS.  16384 rows of 2048 bf16: forward 69 us (4.9
// TB/s of a copy's 5.1), backward 128 us (4.2 TB/s); float32 127 us (5.3) and 245 us (4.4).  Past 4096
// channels the backward's two vectors a thread spill 20 to 25 registers: 16384 rows of 8192 bf16 take
// 1267 us (1.7 TB/s), 8192 rows in float32 867 us (2.5).
#include <algorithm>

#include "sequence.h"

namespace fdc {

template <class T>
constexpr int kNormV = 16 / (int)sizeof(T);  // 16 bytes a lane
constexpr int kBwdV = 4;
// Rows a workgroup takes at once: several only where a row is one wave's (no barrier in between).
template <int TPR>
constexpr int kRows = TPR == 64 ? 4 : 1;

// Sum of v over the TPR threads of a row; every one of them gets it.  red: two halves used in turn,
// so that one barrier a sum is enough.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float *red, int &turn) {
  v = wave_sum(v);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    float *r = red + turn * W;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6] = v;
    __syncthreads();
    v = r[0];
#pragma unroll
    for (int i = 1; i < W; ++i) v += r[i];
  }
  return v;
}

__device__ __forceinline__ float gate_act(int act, float g, float sg) { return act == 0 ? g : act == 1 ? sg : g * sg; }
__device__ __forceinline__ float gate_slope(int act, float g, float sg) {
  return act == 0 ? 1.f : act == 1 ? sg * (1.f - sg) : sg * (1.f + g * (1.f - sg));
}

template <int V>
__device__ __forceinline__ void params(float (&w)[V], const float *p, int c, int nc) {
#pragma unroll
  for (int i = 0; i < V; ++i) w[i] = 1.f;
  if (p != nullptr && nc > 0) {
    const Pack<float, V> x = load_some<float, V>(p + c, nc);
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = x.at(i);
  }
}
template <class T, int V>
__device__ __forceinline__ Pack<T, V> row_part(const T *p, int c, int nc) {
  if (p != nullptr && nc > 0) return load_some<T, V>(p + c, nc);
  return Pack<T, V>{};
}

struct NormOut {
  void *out, *n;
  int64_t out_stride, n_stride;
  float *stats;
};

// The part of a row that a thread holds of `Count` tensors.
template <class T, int V, int NV, int Count>
struct RowParts {
  Pack<T, V> r[Count][NV];
  template <int TPR>
  __device__ __forceinline__ void load(const T *const (&p)[Count], const int64_t (&stride)[Count], int64_t row, int tid,
                                       int D) {
#pragma unroll
    for (int j = 0; j < Count; ++j)
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * TPR + tid) * V;
        r[j][k] = row_part<T, V>(p[j] ? p[j] + row * stride[j] : nullptr, c, D - c);
      }
  }
};

template <class T, int TPR, int NV>
__global__ __launch_bounds__(TPR * kRows<TPR>) void k_block_norm_fwd(fdc_block_norm_args a, NormOut o) {
  constexpr int V = kNormV<T>, RPB = kRows<TPR>;
  __shared__ float red[2 * (TPR / 64)];
  int turn = 0;
  const int tid = threadIdx.x % TPR;
  const int64_t first = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR, step = (int64_t)gridDim.x * RPB;
  const T *const src[3] = {static_cast<const T *>(a.x), static_cast<const T *>(a.f), static_cast<const T *>(a.gate)};
  const int64_t stride[3] = {a.x_stride, a.f_stride, a.gate_stride};
  const float invD = 1.f / (float)a.D;
  const bool has_gate = a.gate != nullptr, normed = a.f != nullptr && a.w_post != nullptr;
  float wp[NV][V], sc[NV][V], w[NV][V];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * TPR + tid) * V;
    params<V>(wp[k], a.w_post, c, a.D - c);
    params<V>(sc[k], a.scale, c, a.D - c);
    params<V>(w[k], a.w_pre, c, a.D - c);
  }
  constexpr bool Ahead = NV == 1;  // two vectors a thread leave no registers for the next row
  RowParts<T, V, NV, 3> in, next;
  if (Ahead && first < a.R) in.template load<TPR>(src, stride, first, tid, a.D);
  for (int64_t row = first; row < a.R; row += step) {
    if (!Ahead)
      in.template load<TPR>(src, stride, row, tid, a.D);
    else if (row + step < a.R)
      next.template load<TPR>(src, stride, row + step, tid, a.D);
    float rf = 1.f, ro = 1.f, s = 0.f;
    if (normed) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) s = fmaf(in.r[1][k].at(i), in.r[1][k].at(i), s);
      rf = 1.f / sqrtf(row_sum<TPR>(s, red, turn) * invD + a.eps);
    }
    float out[NV][V];
    s = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (k * TPR + tid) * V, nc = a.D - c;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float g = in.r[2][k].at(i);
        const float act = has_gate ? gate_act(a.act, g, sigmoid(g)) : 1.f;
        out[k][i] = fmaf(sc[k][i] * act, in.r[1][k].at(i) * rf * wp[k][i], in.r[0][k].at(i));
        s = fmaf(out[k][i], out[k][i], s);
      }
      if (o.out != nullptr && nc > 0) store_some<T, V>(static_cast<T *>(o.out) + row * o.out_stride + c, out[k], nc);
    }
    if (o.n != nullptr) {
      ro = 1.f / sqrtf(row_sum<TPR>(s, red, turn) * invD + a.eps);
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * TPR + tid) * V, nc = a.D - c;
#pragma unroll
        for (int i = 0; i < V; ++i) out[k][i] *= ro * w[k][i];
        if (nc > 0) store_some<T, V>(static_cast<T *>(o.n) + row * o.n_stride + c, out[k], nc);
      }
    }
    if (o.stats != nullptr && tid == 0) {
      o.stats[2 * row] = rf;
      o.stats[2 * row + 1] = ro;
    }
    if (Ahead) in = next;
  }
}

// What a norm's backward leaves of the gradient u of (v r w) by w: (u - vh c) r with vh = v r, c = mean(u vh).
// Of a single channel that is u r (1 - vh^2) = u r (eps r^2), which the difference would lose.
__device__ __forceinline__ float norm_grad(float u, float vh, float r, float c, int D, float eps) {
  return D == 1 ? u * (eps * r * r * r) : fmaf(-vh, c, u) * r;
}

// Rows first, first + step, ...: the sums of the parameters' gradients stay in registers and go to
// part [sharers of a row][3][D] (gscale, gw_post, gw_pre) at the end.
template <class T, int TPR, int NV>
__global__ __launch_bounds__(TPR * kRows<TPR>) void k_block_norm_bwd(fdc_block_norm_args a,
                                                                          fdc_block_norm_grads g,
                                                                          const float *__restrict__ stats,
                                                                          float *__restrict__ part) {
  constexpr int V = kBwdV, RPB = kRows<TPR>;
  __shared__ float red[2 * (TPR / 64)];
  int turn = 0;
  const int tid = threadIdx.x % TPR;
  const int64_t first = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR, step = (int64_t)gridDim.x * RPB;
  const bool has_gate = a.gate != nullptr, normed = a.w_post != nullptr;
  const bool has_n = g.gn != nullptr && a.w_pre != nullptr;
  const T *const src[5] = {static_cast<const T *>(a.x), static_cast<const T *>(a.f), static_cast<const T *>(a.gate),
                           static_cast<const T *>(g.gout), has_n ? static_cast<const T *>(g.gn) : nullptr};
  const int64_t stride[5] = {a.x_stride, a.f_stride, a.gate_stride, g.gout_stride, g.gn_stride};
  const float invD = 1.f / (float)a.D;
  constexpr bool Ahead = NV == 1;  // two vectors a thread leave no registers for the next row or the parameters
  float gscale[NV][V], gpost_w[NV][V], gpre_w[NV][V], wp[V], sc[V], w[V];
  auto load_params = [&](int k) {
    const int c = (k * TPR + tid) * V;
    params<V>(wp, a.w_post, c, a.D - c);
    params<V>(sc, a.scale, c, a.D - c);
    params<V>(w, a.w_pre, c, a.D - c);
  };
  if (Ahead) load_params(0);
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int i = 0; i < V; ++i) gscale[k][i] = gpost_w[k][i] = gpre_w[k][i] = 0.f;
  RowParts<T, V, NV, 5> in, next;
  float2 st = make_float2(1.f, 1.f), next_st = st;
  if (Ahead && first < a.R) {
    in.template load<TPR>(src, stride, first, tid, a.D);
    st = reinterpret_cast<const float2 *>(stats)[first];
  }
  for (int64_t row = first; row < a.R; row += step) {
    if (!Ahead) {
      in.template load<TPR>(src, stride, row, tid, a.D);
      st = reinterpret_cast<const float2 *>(stats)[row];
    } else if (row + step < a.R) {
      next.template load<TPR>(src, stride, row + step, tid, a.D);
      next_st = reinterpret_cast<const float2 *>(stats)[row + step];
    }
    const float rf = st.x, ro = st.y;
    float s = 0.f, go[NV][V], act[NV][V];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      if (!Ahead) load_params(k);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float gv = in.r[2][k].at(i);
        act[k][i] = has_gate ? gate_act(a.act, gv, sigmoid(gv)) : 1.f;
        go[k][i] = fmaf(sc[i] * act[k][i], in.r[1][k].at(i) * rf * wp[i], in.r[0][k].at(i));  // out
        s = fmaf(in.r[4][k].at(i) * w[i], go[k][i] * ro, s);
      }
    }
    const float c1 = has_n ? invD * row_sum<TPR>(s, red, turn) : 0.f;
    float u[NV][V];
    s = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (k * TPR + tid) * V, nc = a.D - c;
      float gg[V];
      if (!Ahead) load_params(k);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float oh = go[k][i] * ro, gnv = in.r[4][k].at(i);
        gpre_w[k][i] = fmaf(gnv, oh, gpre_w[k][i]);
        const float t = in.r[3][k].at(i) + (has_n ? norm_grad(gnv * w[i], oh, ro, c1, a.D, a.eps) : 0.f);
        const float fh = in.r[1][k].at(i) * rf, post = fh * wp[i], gpost = t * sc[i] * act[k][i];
        go[k][i] = t;
        gscale[k][i] = fmaf(t, act[k][i] * post, gscale[k][i]);
        gpost_w[k][i] = fmaf(gpost, fh, gpost_w[k][i]);
        if (has_gate) {
          const float gv = in.r[2][k].at(i);
          gg[i] = t * sc[i] * post * gate_slope(a.act, gv, sigmoid(gv));
        }
        u[k][i] = gpost * wp[i];
        s = fmaf(u[k][i], fh, s);
      }
      if (nc > 0) {
        if (g.gx) store_some<T, V>(static_cast<T *>(g.gx) + row * g.gx_stride + c, go[k], nc);
        if (g.ggate) store_some<T, V>(static_cast<T *>(g.ggate) + row * g.ggate_stride + c, gg, nc);
      }
    }
    if (g.gf) {
      const float c2 = normed ? invD * row_sum<TPR>(s, red, turn) : 0.f;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * TPR + tid) * V, nc = a.D - c;
        if (normed)
#pragma unroll
          for (int i = 0; i < V; ++i) u[k][i] = norm_grad(u[k][i], in.r[1][k].at(i) * rf, rf, c2, a.D, a.eps);
        if (nc > 0) store_some<T, V>(static_cast<T *>(g.gf) + row * g.gf_stride + c, u[k], nc);
      }
    }
    if (Ahead) {
      in = next;
      st = next_st;
    }
  }
  if (part == nullptr) return;
  float *p = part + first * 3 * a.D;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * TPR + tid) * V, nc = a.D - c;
    if (nc <= 0) continue;
    store_some<float, V>(p + c, gscale[k], nc);
    store_some<float, V>(p + a.D + c, gpost_w[k], nc);
    store_some<float, V>(p + 2 * a.D + c, gpre_w[k], nc);
  }
}

namespace {

// f(threads a row, vectors a thread) for rows of `vecs` vectors: as few threads as hold the row, a vector
// each up to 1024 of them.  (Forward vectors are 16 bytes; the backward, which has five rows, three
// parameters and their sums in registers, takes four channels a thread.)
template <int MostNV, class F>
hipError_t by_row(int vecs, F &&f) {
  using std::integral_constant;
#define FDC_ROW(TPR, NV) \
  if (vecs <= TPR * NV) return f(integral_constant<int, TPR>{}, integral_constant<int, NV>{});
  FDC_ROW(64, 1)
  FDC_ROW(128, 1)
  FDC_ROW(256, 1)
  FDC_ROW(512, 1)
  FDC_ROW(1024, 1)
#undef FDC_ROW
  if constexpr (MostNV == 2) return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
  return hipErrorInvalidValue;
}

template <class T>
int fwd_vecs(int D) {
  return (int)ceil_div(D, kNormV<T>);
}
int bwd_vecs(int D) { return (int)ceil_div(D, kBwdV); }
// Workgroups: the forward's fill eight waves a SIMD (the 16-bit forms have registers for five or six, so up
// to two rounds of them); the backward's half of that, by its registers (the float32 form of 512 threads has
// 130 of them, room for one workgroup a compute unit), and because each leaves its sums of the parameters' gradients.
constexpr long long kCus = 256;
long long row_blocks(int64_t R, int rows, int threads, int waves_a_simd) {
  return std::min<long long>(ceil_div(R, rows), kCus * 256 * waves_a_simd / threads);
}
template <int TPR>
long long bwd_blocks(int64_t R) {
  const long long most = row_blocks(R, kRows<TPR>, TPR * kRows<TPR>, 4);
  // four rows each at least, once every compute unit has a workgroup
  return std::min(most, std::max(kCus, ceil_div(R, 4 * kRows<TPR>)));
}

}  // namespace

hipError_t launch_block_norm_fwd(const fdc_block_norm_args &a, void *out, int64_t out_stride, void *n,
                                 int64_t n_stride, float *stats, hipStream_t s) {
  const NormOut o{out, n, out_stride, n_stride, stats};
  return by_dtype(a.dtype, [&](auto tag) {
    using T = decltype(tag);
    return by_row<kNormMaxWidth / (1024 * kNormV<T>)>(fwd_vecs<T>(a.D), [&](auto tpr, auto nv) {
      constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value, RPB = kRows<TPR>;
      const long long blocks = row_blocks(a.R, RPB, TPR * RPB, 8);
      return timed_launch("block_norm_fwd", k_block_norm_fwd<T, TPR, NV>, dim3((unsigned)blocks), dim3(TPR * RPB), 0, s, a,
                          o);
    });
  });
}

size_t block_norm_bwd_ws_floats(int64_t R, int D) {
  size_t n = 0;
  (void)by_row<kNormMaxWidth / (1024 * kBwdV)>(bwd_vecs(D), [&](auto tpr, auto) {
    constexpr int TPR = decltype(tpr)::value, RPB = kRows<TPR>;
    n = (size_t)bwd_blocks<TPR>(R) * RPB * 3 * D;
    return hipSuccess;
  });
  return n;
}

hipError_t launch_block_norm_bwd(const fdc_block_norm_args &a, const float *stats, const fdc_block_norm_grads &g,
                                 float *part, hipStream_t s) {
  float *p = g.gscale || g.gw_post || g.gw_pre ? part : nullptr;
  long long sharers = 0;
  const hipError_t e = by_dtype(a.dtype, [&](auto tag) {
    using T = decltype(tag);
    return by_row<kNormMaxWidth / (1024 * kBwdV)>(bwd_vecs(a.D), [&](auto tpr, auto nv) {
      constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value, RPB = kRows<TPR>;
      const long long blocks = bwd_blocks<TPR>(a.R);
      sharers = blocks * RPB;
      return timed_launch("block_norm_bwd", k_block_norm_bwd<T, TPR, NV>, dim3((unsigned)blocks), dim3(TPR * RPB), 0, s,
                          a, g, stats, p);
    });
  });
  if (e != hipSuccess || p == nullptr) return e;
  ColSegments segs{};
  segs.count = 3;
  float *outs[3] = {g.gscale, g.gw_post, g.gw_pre};
  for (int i = 0; i < 3; ++i) segs.seg[i] = ColSegment{outs[i], a.D, a.D, 1};
  return launch_col_sums(p, sharers, 3LL * a.D, segs, s);
}

}  // namespace fdc
