// Loss of rows of logits against a teacher's top logits (and labels), and its gradient.
//
//   loss = weight ((1 - alpha) (lse1 - z[label]) + alpha tau^2 sum_k q_k (log q_k - (z[idx_k] / tau - lse_tau)))
//   gz[v] = gloss weight ((1 - alpha) (softmax(z)[v] - [v = label]) + alpha tau (softmax(z / tau)[v] - q(v)))
//
// A row needs its largest logit m and the sums s1 = sum exp(z - m), st = sum exp((z - m) / tau), then
// the gradient is elementwise but for the K + 1 places that the teacher and the label name: those
// are written twice, the second time, after a barrier, with their targets subtracted.
// Exponentials and logarithms are taken to base 2 throughout: with c1 = log2(e), ct = log2(e) / tau
// a term is exp2((z - m) c), and the same c stands in every term of the loss, so that its rounding
// is one of the temperature alone.  Logits enter as differences from the row's largest one only, so
// that rows of the type's lowest value (all masked) are uniform and do not overflow.
//
// Many rows: a workgroup holds a row in its registers, as the 16-byte pieces it loaded, so z crosses
// HBM once and gz once.  Few rows, or rows that do not fit: the row is cut into segments, a workgroup
// each, that find their part of m, s1 and st; a wave a row joins them; the gradient is a second pass.
#include <algorithm>

#include "sequence.h"

namespace fdc {

constexpr int kSegThreads = 256;

template <class T>
constexpr int kLogitV = 16 / (int)sizeof(T);

__device__ __forceinline__ float log2_fast(float x) { return __builtin_amdgcn_logf(x); }

// Running maximum m and the sums s1, st relative to it.
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

// The teacher's side of a row: its largest logit and the sum of exp((t - m) / tau) over its entries, 0
// where there are none (or none above -inf); bad: an index or the label lies past the vocabulary.
struct TeacherStat {
  float m, s;
  bool bad;
};

// The K entries of a row's teacher and, as entry K, its label: the place (-1: absent), the teacher's
// logit, the student's logit there, and (written later) the target that the gradient there is less by.
// In dynamic LDS, so that the workgroups of a compute unit are not limited by the largest K.
struct Entries {
  int *place;
  float *t, *z, *target;
  static __host__ __device__ __forceinline__ int padded(int K) { return (K + 4) & ~3; }  // K + 1 and reads of four
  static size_t bytes(int K) { return 16 * (size_t)padded(K); }
  __device__ __forceinline__ Entries(float *lds, int K)
      : place(reinterpret_cast<int *>(lds)), t(lds + padded(K)), z(lds + 2 * padded(K)), target(lds + 3 * padded(K)) {}
};
template <class T>
__device__ __forceinline__ void load_entries(const Entries &en, const fdc_distill_args &a, int64_t row, int tid,
                                             int threads) {
  const T *z = static_cast<const T *>(a.z) + row * a.z_stride;
  for (int k = tid; k <= a.K; k += threads) {
    const int v = k < a.K ? a.idx[row * a.K + k] : a.labels ? a.labels[row] : -1;
    en.place[k] = v;
    en.t[k] = k < a.K ? (float)static_cast<const T *>(a.teacher)[row * a.K + k] : 0.f;
    en.z[k] = v >= 0 && v < a.V ? (float)z[v] : 0.f;
  }
}

// By one wave.
__device__ __forceinline__ TeacherStat teacher_stat(const Entries &en, const fdc_distill_args &a, int lane) {
  const float ct = kLog2e / a.tau;
  TeacherStat te{-INFINITY, 0.f, false};
  int over = 0;
  for (int k = lane; k <= a.K; k += 64) {
    over |= en.place[k] >= a.V;
    if (k < a.K && en.place[k] >= 0) te.m = fmaxf(te.m, en.t[k]);
  }
  te.m = wave_max(te.m);
  te.bad = __any(over);
  // the maximum passes over a NaN, the sum does not
  for (int k = lane; k < a.K; k += 64)
    if (en.place[k] >= 0 && en.t[k] != -INFINITY) te.s += exp2_fast((en.t[k] - te.m) * ct);
  te.s = wave_sum(te.s);
  return te;
}

// By one wave: the loss of a row (of weight other than 0), and its statistics.  In units of two binary
// logarithms, so that a named place at the type's lowest value (masked) stays within float32 like its logit does.
__device__ __forceinline__ void row_loss(const fdc_distill_args &a, int64_t row, int lane, const Entries &en,
                                         const Stat &st, const TeacherStat &te, float *loss, float *stats) {
  const float c1 = 0.5f * kLog2e, ct = kLog2e / a.tau;
  float kl = 0.f;
  if (!te.bad && te.s != 0.f) {
    const float log_st = 0.5f * log2_fast(st.st), log_ts = log2_fast(te.s);
    for (int k = lane; k < a.K; k += 64) {
      if (en.place[k] < 0) continue;
      const float lq = (en.t[k] - te.m) * ct - log_ts, q = exp2_fast(lq);
      if (!(q == 0.f)) kl += q * (0.5f * lq - ((en.z[k] - st.m) * (0.5f * ct) - log_st));
    }
  }
  kl = wave_sum(kl);
  if (lane != 0) return;
  float l = 0.f;
  if (en.place[a.K] >= 0 && !te.bad && a.alpha < 1.f)
    l = (1.f - a.alpha) * (0.5f * log2_fast(st.s1) - (en.z[a.K] - st.m) * c1);
  if (a.alpha > 0.f) l += a.alpha * a.tau * a.tau * kl;
  loss[row] = te.bad ? NAN : (a.weight ? a.weight[row] : 1.f) * (2.f * kLn2) * l;
  float *p = stats + kDistillStats * row;
  p[0] = te.bad ? NAN : st.m;
  p[1] = st.s1, p[2] = st.st, p[3] = te.m, p[4] = te.s;
}
// A row of weight 0, whatever it holds.
__device__ __forceinline__ void row_nothing(int64_t row, int tid, float *loss, float *stats) {
  if (tid == 0) loss[row] = 0.f;
  if (tid < kDistillStats) stats[kDistillStats * row + tid] = 0.f;
}

// The factors of a row's gradient: gz = f1 2^((z - m) c1) + ft 2^((z - m) ct) less the targets' g1
// and gq 2^((t - tm) ct).
struct Factors {
  float c1, ct, m, f1, ft, g1, gq;
  __device__ __forceinline__ Factors(const fdc_distill_args &a, float g, int label, const Stat &st,
                                     const TeacherStat &te) {
    c1 = kLog2e, ct = kLog2e / a.tau;
    m = te.bad ? NAN : st.m;
    g1 = label >= 0 ? g * (1.f - a.alpha) : 0.f;
    const float gt = te.s != 0.f ? g * a.alpha * a.tau : 0.f;
    gq = gt != 0.f ? gt / te.s : 0.f;
    // a row with an index or label past the vocabulary has a NaN maximum
    f1 = m != m ? m : g1 != 0.f ? g1 / st.s1 : 0.f;
    ft = gt != 0.f ? gt / st.st : 0.f;
  }
  // A term that is not wanted is 0, whatever the logit.
  __device__ __forceinline__ float hard(float z) const { return f1 != 0.f ? f1 * exp2_fast((z - m) * c1) : 0.f; }
  __device__ __forceinline__ float soft(float z) const { return ft != 0.f ? ft * exp2_fast((z - m) * ct) : 0.f; }
  // hard(z) + soft(z) where the terms that are wanted are known.
  template <bool Hard, bool Soft>
  __device__ __forceinline__ float sum(float z) const {
    const float d = z - m;
    float o = 0.f;
    if constexpr (Hard) o = f1 * exp2_fast(d * c1);
    if constexpr (Soft) o = fmaf(ft, exp2_fast(d * ct), o);
    return o;
  }
};

// f(hard, soft) as compile-time truth values, for values that are the same in every lane.
template <class F>
__device__ __forceinline__ void by_terms(bool hard, bool soft, F &&f) {
  using std::bool_constant;
  if (__builtin_amdgcn_readfirstlane(hard)) {
    if (__builtin_amdgcn_readfirstlane(soft))
      f(bool_constant<true>{}, bool_constant<true>{});
    else
      f(bool_constant<true>{}, bool_constant<false>{});
  } else {
    if (__builtin_amdgcn_readfirstlane(soft))
      f(bool_constant<false>{}, bool_constant<true>{});
    else
      f(bool_constant<false>{}, bool_constant<false>{});
  }
}

// The targets of a row's entries (a barrier before write_entries), and of the padding that it reads.
__device__ __forceinline__ void put_targets(const Entries &en, const Factors &f, int K, float tm, int tid, int threads) {
  for (int k = tid; k < Entries::padded(K); k += threads)
    en.target[k] = k < K && en.place[k] >= 0 && f.gq != 0.f ? f.gq * exp2_fast((en.t[k] - tm) * f.ct) : 0.f;
}
// The gradient at the entries within [begin, end), by threads that stand for an entry each (the
// first of those that name the same place writes it).  Each term's probability and its targets are
// subtracted before the terms are added: both may be close to 1.
template <class T>
__device__ __forceinline__ void write_entries(const Entries &en, const Factors &f, int K, T *gz, int begin, int end,
                                              int tid, int threads) {
  for (int k = tid; k <= K; k += threads) {
    const int v = en.place[k];
    if (v < begin || v >= end) continue;
    float hard = f.hard(en.z[k]), soft = f.soft(en.z[k]);
    bool first = true;
#pragma unroll 4
    for (int j = 0; j < K; j += 4) {
      const int4 at = *reinterpret_cast<const int4 *>(&en.place[j]);
      const float4 q = *reinterpret_cast<const float4 *>(&en.target[j]);
      const int p[4] = {at.x, at.y, at.z, at.w};
      const float t[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool same = p[i] == v && j + i < K;
        soft -= same ? t[i] : 0.f;
        first = first && !(same && j + i < k);
      }
    }
    if (en.place[K] == v) hard -= f.g1;
    if (first) gz[v] = (T)(hard + soft);
  }
}

// ---- a row a workgroup -------------------------------------------------------
// Keeps the compiler from holding the floats of one pass over a row's pieces for the next: 16-bit
// logits would take twice their registers, and fewer rows would be in flight on a compute unit
// (for float32 it only costs: 2048 x 32000 206 us with it, 166 us without).  For float16 rows of 8 pieces
// it does not hold: the gradient's form spills 164 registers (bfloat16's 5), and 4096 x 32000 takes 497 us
// where bfloat16 takes 153.
template <class T, int V>
__device__ __forceinline__ void keep_packed(Pack<T, V> &x) {
  if constexpr (sizeof(T) == 2) asm volatile("" : "+v"(x.w[0]), "+v"(x.w[1]), "+v"(x.w[2]), "+v"(x.w[3]));
}

// A workgroup a row.  The row's phases (load, largest logit, sums, gradient) follow each other behind
// barriers; the rows on a compute unit overlap them: 512 threads are two waves a SIMD, so that four rows of 4
// pieces (f16: three), three of 8, and of 16 pieces two in 16 bits and one in float32 (168 registers) fit at once.  4096 x 32000
// bfloat16, K = 64: 153 us (3.4 TB/s of 5.1; its 15 plain operations and four exponentials an element would take
// 87 us alone); 2048 x 32000 float32 163 us (3.2).  Measured
// and not kept: workgroups that take row after row with the next one loaded ahead (200 to 220 us: twice the
// registers, half the rows in flight), 256 threads (185), 1024 threads (262).
template <class T, int TH, int NV, bool Grad>
__global__ __launch_bounds__(TH, NV == 16 ? (sizeof(T) == 4 ? 3 : 4) : NV == 8 ? 6 : 1) void k_distill_row(fdc_distill_args a,
                                                                                    float *__restrict__ loss,
                                                                                    float *__restrict__ stats,
                                                                                    const float *__restrict__ gloss,
                                                                                    void *gz_, int64_t gz_stride) {
  constexpr int V = kLogitV<T>, W = TH / 64;
  extern __shared__ __align__(16) float lds[];
  const Entries en(lds, a.K);
  __shared__ float rmax[W], rs1[W], rst[W];
  __shared__ TeacherStat te;
  const int64_t row = (int64_t)blockIdx.y * 32768 + blockIdx.x;
  if (row >= a.R) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float c1 = kLog2e, ct = kLog2e / a.tau;
  const T *z = static_cast<const T *>(a.z) + row * a.z_stride;
  T *gz = Grad ? static_cast<T *>(gz_) + row * gz_stride : nullptr;
  const float up = Grad ? gloss[row] : 0.f, weight = a.weight ? a.weight[row] : 1.f;
  if (weight == 0.f) {
    row_nothing(row, tid, loss, stats);
    if constexpr (Grad) {
      const float o[V] = {};
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * TH + tid) * V;
        if (c < a.V) store_some<T, V>(gz + c, o, a.V - c);
      }
    }
    return;
  }
  Pack<T, V> x[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * TH + tid) * V, n = a.V - c;
    if (n > 0) {
      x[k] = load_some<T, V>(z + c, n, -INFINITY);
    } else {
      const unsigned none = element_bits<T>((T)-INFINITY);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[k].w[i] = sizeof(T) == 4 ? none : none | none << 16;
    }
  }
  load_entries<T>(en, a, row, tid, TH);
  Stat st{-INFINITY, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int i = 0; i < V; ++i) st.m = fmaxf(st.m, x[k].at(i));
  st.m = wave_max(st.m);
  if (lane == 0) rmax[wave] = st.m;
#pragma unroll
  for (int k = 0; k < NV; ++k) keep_packed(x[k]);
  __syncthreads();
#pragma unroll
  for (int w = 0; w < W; ++w) st.m = fmaxf(st.m, rmax[w]);
  if (wave == W - 1) {
    const TeacherStat t = teacher_stat(en, a, lane);
    if (lane == 0) te = t;
  }
  by_terms(en.place[a.K] >= 0 && a.alpha < 1.f, a.alpha > 0.f, [&](auto hard, auto soft) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d = x[k].at(i) - st.m;
        if constexpr (hard.value) st.s1 += exp2_fast(d * c1);
        if constexpr (soft.value) st.st += exp2_fast(d * ct);
      }
      if constexpr (sizeof(T) == 2) __builtin_amdgcn_sched_barrier(0);  // a piece at a time: its floats die with it
    }
  });
  st.s1 = wave_sum(st.s1);
  st.st = wave_sum(st.st);
  if (lane == 0) rs1[wave] = st.s1, rst[wave] = st.st;
  __syncthreads();
  st.s1 = st.st = 0.f;
#pragma unroll
  for (int w = 0; w < W; ++w) st.s1 += rs1[w], st.st += rst[w];
  if constexpr (Grad) {
#pragma unroll
    for (int k = 0; k < NV; ++k) keep_packed(x[k]);
    const Factors f(a, up * weight, en.place[a.K], st, te);
    put_targets(en, f, a.K, te.m, tid, TH);
    by_terms(f.f1 != 0.f, f.ft != 0.f, [&](auto hard, auto soft) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * TH + tid) * V;
        float o[V];
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] = f.template sum<hard.value, soft.value>(x[k].at(i));
        if (c < a.V) store_some<T, V>(gz + c, o, a.V - c);
        __builtin_amdgcn_sched_barrier(0);
      }
    });
    __syncthreads();
    write_entries<T>(en, f, a.K, gz, 0, a.V, tid, TH);
  }
  // the first waves write the entries, the last one does what a wave does alone
  if (wave == W - 1) row_loss(a, row, lane, en, st, te, loss, stats);
}

// ---- a row in segments ---------------------------------------------------------
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
        if (i < n) m = fmaxf(m, x.at(i));
      st.s1 *= rescale(st.m, m, c1);
      st.st *= rescale(st.m, m, ct);
      st.m = m;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d = x.at(i) - m;  // NaN where the row holds -inf alone so far
        const bool none = i >= n || x.at(i) == -INFINITY;
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

// A wave a row: its segments in order, then the loss.
template <class T>
__global__ __launch_bounds__(64) void k_distill_join(fdc_distill_args a, const float *__restrict__ part, int segs,
                                                     float *__restrict__ loss, float *__restrict__ stats) {
  extern __shared__ __align__(16) float lds[];
  const Entries en(lds, a.K);
  const int lane = threadIdx.x;
  const int64_t row = (int64_t)blockIdx.y * 32768 + blockIdx.x;
  if (row >= a.R) return;
  const float c1 = kLog2e, ct = kLog2e / a.tau;
  if (a.weight && a.weight[row] == 0.f) {
    row_nothing(row, lane, loss, stats);
    return;
  }
  load_entries<T>(en, a, row, lane, 64);
  Stat st{-INFINITY, 0.f, 0.f};
  for (int i = lane; i < segs; i += 64) {
    const float *p = part + (row * segs + i) * 3;
    join(st, Stat{p[0], p[1], p[2]}, c1, ct);
  }
  st = wave_join(st, c1, ct);
  __syncthreads();
  row_loss(a, row, lane, en, st, teacher_stat(en, a, lane), loss, stats);
}

// Segment blockIdx.x of row blockIdx.y of the gradient.  z and gz may be the same memory: a thread
// reads the logits it writes the gradients of, and the entries' are read before.
template <class T>
__global__ __launch_bounds__(kSegThreads) void k_distill_grad(fdc_distill_args a, const float *__restrict__ stats,
                                                              const float *__restrict__ gloss, void *gz_,
                                                              int64_t gz_stride, int seg) {
  constexpr int V = kLogitV<T>;
  extern __shared__ __align__(16) float lds[];
  const Entries en(lds, a.K);
  const int64_t row = (int64_t)blockIdx.y + (int64_t)blockIdx.z * 32768;
  if (row >= a.R) return;
  const T *z = static_cast<const T *>(a.z) + row * a.z_stride;
  T *gz = static_cast<T *>(gz_) + row * gz_stride;
  const float weight = a.weight ? a.weight[row] : 1.f;
  const float *p = stats + kDistillStats * row;
  const Stat st{p[0], p[1], p[2]};
  const TeacherStat te{p[3], p[4], false};
  const Factors f(a, weight == 0.f ? 0.f : gloss[row] * weight, a.labels ? a.labels[row] : -1, st, te);
  const int begin = blockIdx.x * seg, end = min(a.V, begin + seg);
  load_entries<T>(en, a, row, threadIdx.x, kSegThreads);
  __syncthreads();
  put_targets(en, f, a.K, te.m, threadIdx.x, kSegThreads);
  by_terms(f.f1 != 0.f, f.ft != 0.f, [&](auto hard, auto soft) {
    for (int c = begin + threadIdx.x * V; c < end; c += kSegThreads * V) {
      const int n = min(V, end - c);
      const Pack<T, V> x = load_some<T, V>(z + c, n);
      float o[V];
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = f.template sum<hard.value, soft.value>(x.at(i));
      store_some<T, V>(gz + c, o, n);
    }
  });
  __syncthreads();
  if (weight != 0.f) write_entries<T>(en, f, a.K, gz, begin, end, threadIdx.x, kSegThreads);
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
dim3 segment_grid(const Segments &sg, int64_t R) {
  return dim3((unsigned)sg.segs, (unsigned)std::min<int64_t>(R, 32768), (unsigned)ceil_div(R, 32768));
}
dim3 row_grid(int64_t R) { return dim3((unsigned)std::min<int64_t>(R, 32768), (unsigned)ceil_div(R, 32768)); }

// Rows that fit a workgroup's registers (16 pieces of 16 bytes in 512 threads), and enough of them for
// the chip's 256 compute units: one for each, or three where a row takes a third of a unit's registers or more.
// Loss and gradient in segments (a row fewer) and a row a workgroup: 256 rows of 8192 bf16 19.5 and 13.0 us, f32
// 21.9 and 13.4; 768 rows of 20000 bf16 42 and 26, f32 48 and 43; of 60000 bf16 76 and 56.  f16 is as bf16 but for
// rows of 5 to 8 pieces, whose spills (see keep_packed) make the row a workgroup the slower one: 20000 logits 43
// and 74 us.  Longer rows are read twice: 1024 of 65536 bf16 75 us, of 65537 107 us.
bool whole_rows(int dtype, int64_t R, int V) {
  const long long pieces = ceil_div(V, 16 / (int)dtype_size(dtype));
  return pieces <= 512 * 16 && R >= (pieces <= 512 * 4 ? 256 : 3 * 256);
}

// f(threads, pieces a thread) for rows of `vecs` 16-byte pieces (at most 512 * 16).
template <class F>
hipError_t by_pieces(long long vecs, F &&f) {
  using std::integral_constant;
#define FDC_ROW(TH, NV) \
  if (vecs <= TH * NV) return f(integral_constant<int, TH>{}, integral_constant<int, NV>{});
  FDC_ROW(64, 1)
  FDC_ROW(128, 2)
  FDC_ROW(256, 4)
  FDC_ROW(512, 4)
  FDC_ROW(512, 8)
#undef FDC_ROW
  return f(integral_constant<int, 512>{}, integral_constant<int, 16>{});
}

}  // namespace

size_t distill_ws_floats(int dtype, int64_t R, int V) {
  return whole_rows(dtype, R, V) ? 0 : (size_t)R * segments(dtype, R, V).segs * 3;
}

hipError_t launch_distill(const fdc_distill_args &a, float *loss, float *stats, const float *gloss, void *gz,
                          int64_t gz_stride, float *ws, hipStream_t s) {
  return by_dtype(a.dtype, [&](auto tag) {
    using T = decltype(tag);
    if (whole_rows(a.dtype, a.R, a.V))
      return by_pieces(ceil_div(a.V, kLogitV<T>), [&](auto threads, auto pieces) {
        constexpr int TH = decltype(threads)::value, NV = decltype(pieces)::value;
        if (gz != nullptr)
          return timed_launch("distill_row_grad", k_distill_row<T, TH, NV, true>, row_grid(a.R), dim3(TH),
                              Entries::bytes(a.K), s, a, loss, stats, gloss, gz, gz_stride);
        return timed_launch("distill_row", k_distill_row<T, TH, NV, false>, row_grid(a.R), dim3(TH), Entries::bytes(a.K),
                            s, a, loss, stats, gloss, gz, gz_stride);
      });
    const Segments sg = segments(a.dtype, a.R, a.V);
    if (hipError_t e = timed_launch("distill_part", k_distill_part<T>, segment_grid(sg, a.R), dim3(kSegThreads), 0, s, a,
                                    ws, sg.seg, sg.segs))
      return e;
    if (hipError_t e = timed_launch("distill_join", k_distill_join<T>, row_grid(a.R), dim3(64), Entries::bytes(a.K), s, a,
                                    (const float *)ws, sg.segs, loss, stats))
      return e;
    return gz != nullptr ? launch_distill_bwd(a, stats, gloss, gz, gz_stride, s) : hipSuccess;
  });
}

hipError_t launch_distill_bwd(const fdc_distill_args &a, const float *stats, const float *gloss, void *gz,
                              int64_t gz_stride, hipStream_t s) {
  const Segments sg = segments(a.dtype, a.R, a.V);
  return by_dtype(a.dtype, [&](auto tag) {
    using T = decltype(tag);
    return timed_launch("distill_grad", k_distill_grad<T>, segment_grid(sg, a.R), dim3(kSegThreads), Entries::bytes(a.K), s, a, stats, gloss,
                        gz, gz_stride, sg.seg);
  });
}

}  // namespace fdc
