// Loss of rows of logits against a teacher's top logits (and labels), and its gradient.
//
//   loss = weight ((1 - alpha) (lse1 - z[label]) + alpha tau^2 sum_k q_k (log q_k - (z[idx_k] / tau - lse_tau)))
//   gz[v] = gloss weight ((1 - alpha) (softmax(z)[v] - [v = label]) + alpha tau (softmax(z / tau)[v] - q(v)))
//
// One pass over a row finds its largest logit and the sums of exp(z - max) and exp((z - max) / tau)
// together.  A row is cut into segments, a workgroup each, so that few rows still use the whole
// chip; a wave a row joins them and adds the teacher's terms.  The gradient is a second pass; the few
// entries that the teacher or the label takes part in are found by a bitmap of their places.
// Bound by HBM where a row holds two exponentials an element: 2 bytes read, 2 written.
#include <algorithm>

#include "sequence.h"

namespace fdc {

constexpr int kSegThreads = 256;

template <class T>
constexpr int kLogitV = 16 / (int)sizeof(T);

// Running maximum m and the sums s1 = sum exp(z - m), st = sum exp((z - m) / tau).
struct Stat {
  float m, s1, st;
};
// What a sum relative to m is multiplied with to be relative to `to` >= m (m = -inf: the sum is 0).
__device__ __forceinline__ float rescale(float m, float to, float c) {
  return m == to ? 1.f : exp2_fast((m - to) * c);
}
__device__ __forceinline__ void join(Stat &a, const Stat &b, float c1, float ct) {
  const float m = fmaxf(a.m, b.m);
  a.s1 = a.s1 * rescale(a.m, m, c1) + b.s1 * rescale(b.m, m, c1);
  a.st = a.st * rescale(a.m, m, ct) + b.st * rescale(b.m, m, ct);
  a.m = m;
}
__device__ __forceinline__ Stat wave_join(Stat a, float c1, float ct) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const Stat b{__shfl_xor(a.m, off, 64), __shfl_xor(a.s1, off, 64), __shfl_xor(a.st, off, 64)};
    join(a, b, c1, ct);
  }
  return a;
}

// Segment blockIdx.x of row blockIdx.y -> part[row][segment].
template <class T>
__global__ __launch_bounds__(kSegThreads) void k_distill_part(fdc_distill_args a, float *__restrict__ part, int seg,
                                                              int segs) {
  constexpr int V = kLogitV<T>;
  __shared__ Stat red[kSegThreads / 64];
  const int64_t row = (int64_t)blockIdx.y + (int64_t)blockIdx.z * 32768;
  if (row >= a.R) return;
  const float c1 = kLog2e, ct = kLog2e / a.tau;
  const T *z = static_cast<const T *>(a.z) + row * a.z_stride;
  const int end = min(a.V, ((int)blockIdx.x + 1) * seg);
  Stat st{-INFINITY, 0.f, 0.f};
  if (a.weight == nullptr || a.weight[row] != 0.f) {
    for (int c = blockIdx.x * seg + threadIdx.x * V; c < end; c += kSegThreads * V) {
      const int n = min(V, end - c);
      const Pack<T, V> x = load_some<T, V>(z + c, n);
      float m = st.m;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i < n) m = fmaxf(m, (float)x.v[i]);
      st.s1 *= rescale(st.m, m, c1);
      st.st *= rescale(st.m, m, ct);
      st.m = m;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d = (float)x.v[i] - m;  // NaN where the row holds -inf alone so far
        const bool none = i >= n || (float)x.v[i] == -INFINITY;
        st.s1 += none ? 0.f : exp2_fast(d * c1);
        st.st += none ? 0.f : exp2_fast(d * ct);
      }
    }
  }
  st = wave_join(st, c1, ct);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = st;
  __syncthreads();
  if (threadIdx.x != 0) return;
#pragma unroll
  for (int w = 1; w < kSegThreads / 64; ++w) join(st, red[w], c1, ct);
  float *p = part + (row * segs + blockIdx.x) * 3;
  p[0] = st.m, p[1] = st.s1, p[2] = st.st;
}

// The teacher's side of a row for one wave: q_k = exp(t_k - lse) with lse = logsumexp(teacher / tau),
// -inf where the row has no entry; `bad`: an index past the vocabulary.
template <class T>
struct Teacher {
  const int *idx;
  const T *t;
  float lse;
  bool bad;
  __device__ __forceinline__ Teacher(const fdc_distill_args &a, int64_t row, int lane) {
    idx = a.idx + row * a.K;
    t = static_cast<const T *>(a.teacher) + row * a.K;
    float m = -INFINITY, s = 0.f;
    int over = 0;
    for (int k = lane; k < a.K; k += 64) {
      if (idx[k] >= a.V) over = 1;
      if (idx[k] >= 0) m = fmaxf(m, (float)t[k] / a.tau);
    }
    m = wave_max(m);
    bad = __any(over);
    for (int k = lane; k < a.K; k += 64)
      if (idx[k] >= 0 && m != -INFINITY) s += exp_fast((float)t[k] / a.tau - m);
    s = wave_sum(s);
    lse = m == -INFINITY ? m : m + kLn2 * __builtin_amdgcn_logf(s);
  }
};

// The loss of a row from its sums, by one wave.
template <class T>
__device__ __forceinline__ void row_loss(const fdc_distill_args &a, int64_t row, int lane, Stat st, float *loss,
                                         float *stats) {
  const float weight = a.weight ? a.weight[row] : 1.f;
  if (weight == 0.f) {
    if (lane == 0) loss[row] = 0.f;
    if (lane < 4) stats[4 * row + lane] = 0.f;
    return;
  }
  const Teacher<T> te(a, row, lane);
  const T *z = static_cast<const T *>(a.z) + row * a.z_stride;
  const int label = a.labels ? a.labels[row] : -1;
  const float lse1 = st.m + kLn2 * __builtin_amdgcn_logf(st.s1);
  const float lset = st.m / a.tau + kLn2 * __builtin_amdgcn_logf(st.st);
  const bool bad = te.bad || label >= a.V;
  float kl = 0.f;
  if (!bad && te.lse != -INFINITY)
    for (int k = lane; k < a.K; k += 64) {
      const int i = te.idx[k];
      if (i < 0) continue;
      const float lq = (float)te.t[k] / a.tau - te.lse;
      const float q = exp_fast(lq);
      if (!(q == 0.f)) kl += q * (lq - ((float)z[i] / a.tau - lset));
    }
  kl = wave_sum(kl);
  if (lane != 0) return;
  float l = 0.f;
  if (label >= 0 && !bad && a.alpha < 1.f) l = (1.f - a.alpha) * (lse1 - (float)z[label]);
  if (a.alpha > 0.f) l += a.alpha * a.tau * a.tau * kl;
  loss[row] = bad ? NAN : weight * l;
  stats[4 * row] = bad ? NAN : st.m;
  stats[4 * row + 1] = st.s1;
  stats[4 * row + 2] = st.st;
  stats[4 * row + 3] = te.lse;
}

// A wave a row: its segments in order, then the loss.
template <class T>
__global__ __launch_bounds__(256) void k_distill_join(fdc_distill_args a, const float *__restrict__ part, int segs,
                                                      float *__restrict__ loss, float *__restrict__ stats) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.R) return;
  const float c1 = kLog2e, ct = kLog2e / a.tau;
  Stat st{-INFINITY, 0.f, 0.f};
  for (int i = lane; i < segs; i += 64) {
    const float *p = part + (row * segs + i) * 3;
    join(st, Stat{p[0], p[1], p[2]}, c1, ct);
  }
  st = wave_join(st, c1, ct);
  row_loss<T>(a, row, lane, st, loss, stats);
}

// Places of a row that the teacher or the label takes part in: bit (v / 8) mod kMapBits of `map`
// says that one of the eight logits v .. v + 7 may be such a place.
constexpr int kMapBits = 16384;

// Segment blockIdx.x of row blockIdx.y of the gradient.  z and gz may be the same memory: a thread
// reads the logits it writes the gradients of, and no others.
template <class T>
__global__ __launch_bounds__(kSegThreads) void k_distill_grad(fdc_distill_args a, const float *__restrict__ stats,
                                                              const float *__restrict__ gloss, void *gz_,
                                                              int64_t gz_stride, int seg) {
  constexpr int V = kLogitV<T>;
  __shared__ unsigned map[kMapBits / 32];
  __shared__ int place[kDistillMaxTeacher];
  __shared__ float q[kDistillMaxTeacher];
  const int64_t row = (int64_t)blockIdx.y + (int64_t)blockIdx.z * 32768;
  if (row >= a.R) return;
  const T *z = static_cast<const T *>(a.z) + row * a.z_stride;
  T *gz = static_cast<T *>(gz_) + row * gz_stride;
  const float weight = a.weight ? a.weight[row] : 1.f;
  const float m = stats[4 * row], s1 = stats[4 * row + 1], st = stats[4 * row + 2], lse = stats[4 * row + 3];
  const int label = a.labels ? a.labels[row] : -1;
  const float g = weight == 0.f ? 0.f : gloss[row] * weight;
  const float g1 = label >= 0 ? g * (1.f - a.alpha) : 0.f, gt = lse != -INFINITY ? g * a.alpha * a.tau : 0.f;
  const int begin = blockIdx.x * seg, end = min(a.V, begin + seg);
  for (int i = threadIdx.x; i < kMapBits / 32; i += kSegThreads) map[i] = 0;
  __syncthreads();
  if (gt != 0.f)
    for (int k = threadIdx.x; k < a.K; k += kSegThreads) {
      const int v = a.idx[row * a.K + k];
      place[k] = v;
      q[k] = v >= 0 ? gt * exp_fast((float)static_cast<const T *>(a.teacher)[row * a.K + k] / a.tau - lse) : 0.f;
      if (v >= begin && v < end) {
        const int bit = (v - begin) / V % kMapBits;
        atomicOr(&map[bit / 32], 1u << (bit % 32));
      }
    }
  if (threadIdx.x == 0 && g1 != 0.f && label >= begin && label < end) {
    const int bit = (label - begin) / V % kMapBits;
    atomicOr(&map[bit / 32], 1u << (bit % 32));
  }
  __syncthreads();
  const float c1 = kLog2e, ct = kLog2e / a.tau;
  // a row with an index or label past the vocabulary has a NaN maximum
  const float f1 = m != m ? m : g1 != 0.f ? g1 / s1 : 0.f, ft = gt != 0.f ? gt / st : 0.f;
  for (int c = begin + threadIdx.x * V; c < end; c += kSegThreads * V) {
    const int n = min(V, end - c);
    const Pack<T, V> x = load_some<T, V>(z + c, n);
    float o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float d = (float)x.v[i] - m;
      o[i] = f1 != 0.f ? f1 * exp2_fast(d * c1) : 0.f;
      if (ft != 0.f) o[i] = fmaf(ft, exp2_fast(d * ct), o[i]);
    }
    const int bit = (c - begin) / V % kMapBits;
    if (map[bit / 32] >> (bit % 32) & 1) {
      // each term's probability and its target are subtracted before the terms are added: both may be
      // close to 1
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d = (float)x.v[i] - m;
        float hard = f1 != 0.f ? f1 * exp2_fast(d * c1) : 0.f, soft = ft != 0.f ? ft * exp2_fast(d * ct) : 0.f;
        if (g1 != 0.f && label == c + i) hard -= g1;
        if (gt != 0.f)
          for (int k = 0; k < a.K; ++k)
            if (place[k] == c + i) soft -= q[k];
        o[i] = hard + soft;
      }
    }
    store_some<T, V>(gz + c, o, n);
  }
}

namespace {

struct Segments {
  int seg, segs;
};
// Segments long enough to amortise a workgroup's start, short enough that few rows fill the chip.
Segments segments(int dtype, int64_t R, int V) {
  const int unit = kSegThreads * 16 / (int)dtype_size(dtype);
  long long per = ceil_div(V, unit);  // passes of a workgroup over the whole row
  while (per > 1 && R * ceil_div(V, per * unit) < 2048) per = ceil_div(per, 2);
  Segments s;
  s.seg = (int)(per * unit);
  s.segs = (int)ceil_div(V, s.seg);
  return s;
}
dim3 row_grid(const Segments &sg, int64_t R) {
  const int64_t y = std::min<int64_t>(R, 32768);
  return dim3((unsigned)sg.segs, (unsigned)y, (unsigned)ceil_div(R, 32768));
}

}  // namespace

size_t distill_ws_floats(int dtype, int64_t R, int V) { return (size_t)R * segments(dtype, R, V).segs * 3; }

hipError_t launch_distill(const fdc_distill_args &a, float *loss, float *stats, const float *gloss, void *gz,
                          int64_t gz_stride, float *ws, hipStream_t s) {
  const Segments sg = segments(a.dtype, a.R, a.V);
  const hipError_t e = by_dtype(a.dtype, [&](auto tag) {
    using T = decltype(tag);
    if (hipError_t e = timed_launch("distill_part", k_distill_part<T>, row_grid(sg, a.R), dim3(kSegThreads), 0, s, a, ws,
                                    sg.seg, sg.segs))
      return e;
    return timed_launch("distill_join", k_distill_join<T>, dim3((unsigned)ceil_div(a.R, 4)), dim3(256), 0, s, a,
                        (const float *)ws, sg.segs, loss, stats);
  });
  if (e != hipSuccess || gz == nullptr) return e;
  return launch_distill_bwd(a, stats, gloss, gz, gz_stride, s);
}

hipError_t launch_distill_bwd(const fdc_distill_args &a, const float *stats, const float *gloss, void *gz,
                              int64_t gz_stride, hipStream_t s) {
  const Segments sg = segments(a.dtype, a.R, a.V);
  return by_dtype(a.dtype, [&](auto tag) {
    using T = decltype(tag);
    return timed_launch("distill_grad", k_distill_grad<T>, row_grid(sg, a.R), dim3(kSegThreads), 0, s, a, stats, gloss, gz,
                        gz_stride, sg.seg);
  });
}

}  // namespace fdc
