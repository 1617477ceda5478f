// Cross attention: the forward for few rows a key head (a single token of each sequence, above all).
#include "cross_attention.h"

namespace fdc {

using namespace attention;

namespace {

// A workgroup has a key head's rows, at most 32, and a run of its keys; its waves take blocks of 32 keys in turn, each on
// its own: k and v are read once, a block ahead of the products (HBM-bound: 64 x 4096 keys of 8 heads of 128 f16, 1.07 GB in
// 215 us, 5.0 TB/s; 1024 keys of 16 heads of 64 bf16 take 10.7 us, latencies alone, in one launch where runs and their join took
// 13.8 in two), and pass through the wave's own rows of LDS without barriers.  At the end the waves' maxima, sums and outputs are joined in LDS,
// in wave order, so that a call is one launch where there are sequences enough or keys few enough.  16-bit heads of 128
// channels have 29 registers spilled, those of 96 8.
template <class T, int DP, int W>
constexpr size_t few_lds(int rows) {
  const size_t areas = (size_t)32 * W * kStride<T, DP> * sizeof(T), outs = (size_t)W * rows * DP * sizeof(float);
  return std::max(areas, outs) + (size_t)3 * W * 32 * sizeof(float);
}
template <class T, int DP, int W>
__global__ __launch_bounds__(64 * W) void k_attn_few(Attn p, float *__restrict__ part, int splits, int run, int lds_stats) {
  constexpr int V = 16 / (int)sizeof(T), PR = DP / V, N = 32 * PR / 64, S = kStride<T, DP>;
  extern __shared__ __align__(16) char lds_[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  const int split = blockIdx.x % splits, bg = blockIdx.x / splits, b = bg / p.a.G, g = bg - b * p.a.G;
  const int keys = length_of(p.a.lengths, b, p.a.Lk), queries = length_of(p.a.q_lengths, b, p.a.Lq);
  T *area = reinterpret_cast<T *>(lds_) + wave * 32 * S;
  const Row row = row_of(p, g, lane & 31, queries);
  WaveRows<T, DP> wq;
  wq.issue(static_cast<const T *>(p.a.q.p), offset_of(p.a.q, b, row.t, row.head), p.a.D, p.wide, row.live, lane);
  v16f o[DP / 32] = {};
  float m = -INFINITY, l = 0.f, w = 0.f;  // the sum, and that of the rounded probabilities
  const int first = split * run, last = min(first + run, (keys + 31) / 32);
  Pack<T, V> xk[N], xv[N];
  auto load = [&](Pack<T, V>(&x)[N], const fdc_heads &h, int block, uint64_t there) {
    const T *base = at<T>(h, b, (int64_t)block * 32, g);
    const int most = p.a.Lk - 1 - block * 32;
    if (p.wide) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int r = (lane + 64 * i) / PR, c = (lane + 64 * i) % PR * V;
        x[i] = load_pack<T, V>(base + min(r, most) * h.token_stride + first_of<T>(c, p.a.D));
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int r = (lane + 64 * i) / PR, c = (lane + 64 * i) % PR * V;
        x[i] = Pack<T, V>{};
        if (c < p.a.D && (there >> r & 1)) x[i] = load_some<T, V>(base + r * h.token_stride + c, p.a.D - c);
      }
    }
  };
  auto put = [&](Pack<T, V>(&x)[N], uint64_t there) {
    move_pieces(x, p.a.D, [&](int i) { return (lane + 64 * i) % PR * V; });
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = (lane + 64 * i) / PR, c = (lane + 64 * i) % PR * V;
      if (!(there >> r & 1) || c >= p.a.D) x[i] = Pack<T, V>{};
      *reinterpret_cast<Pack<T, V> *>(area + r * S + c) = x[i];
    }
    wave_sync();
  };
  int block = first + wave;
  uint64_t there = 0;
  if (block < last) {
    there = keys_there(p, b, block * 32, keys, lane, 32);
    load(xk, p.a.k, block, there);
    load(xv, p.a.v, block, there);
  }
  Frag<T> q[DP / 16];
  wq.land(q, area, p.a.D, row.live, lane);
  for (; block < last; block += W) {
    const bool more = block + W < last;
    const uint64_t next = more ? keys_there(p, b, (block + W) * 32, keys, lane, 32) : 0;
    put(xk, there);
    if (more) load(xk, p.a.k, block + W, next);
    v16f s = {};
    {
      Rows<T, DP, DP / 16> rows;
      rows.load(area, 0, 0, lane);
#pragma unroll
      for (int i = 0; i < DP / 16; ++i) mma(s, rows.f[i], q[i]);
    }
    wave_sync();
    put(xv, there);
    if (more) load(xv, p.a.v, block + W, next);
    if (there != 0xffffffffull) {
      const uint64_t mine = there >> (4 * half);
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (!(mine >> (8 * (j / 4) + j % 4) & 1)) s[j] = -INFINITY;
    }
    float top = s[0];
#pragma unroll
    for (int j = 1; j < 16; ++j) top = fmaxf(top, s[j]);
    top = halves_max(top) * p.c;
    const bool late = top > m + kLate;
    if (__any(late)) {
      const float to = late ? top : m, f = m == to ? 1.f : exp2_fast(m - to);
      l *= f, w *= f;
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) o[d] *= f;
      m = to;
    }
    const float base = kUp<T> - (m == -INFINITY ? 0.f : m);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      s[j] = exp2_fast(fmaf(s[j], p.c, base));
      l += s[j];
    }
    const Frag<T> e[2] = {score_frag<T>(s, 0), score_frag<T>(s, 1)};
    if constexpr (sizeof(T) == 2) w = add_values(e[1], add_values(e[0], w));
    Columns<T, DP> cols;
    cols.load(area, 0, lane);
    cols.add_to(o, e);
    wave_sync();
    there = next;
  }
  // the waves' results of a row, relative to the largest maximum
  float *stats = reinterpret_cast<float *>(lds_ + lds_stats), *outs = reinterpret_cast<float *>(lds_);
  l = halves_sum(l);
  w = sizeof(T) == 2 ? halves_sum(w) : l;
  if (half == 0) {
    float *to = stats + (wave * 32 + lane) * 3;
    to[0] = m, to[1] = l, to[2] = w;
  }
  __syncthreads();
  float most = -INFINITY;
#pragma unroll
  for (int i = 0; i < W; ++i) most = fmaxf(most, stats[(i * 32 + (lane & 31)) * 3]);
  if ((lane & 31) < p.R) {
    float *to = outs + ((size_t)wave * p.R + (lane & 31)) * DP;
    each_four<DP>(o, DP, half, m == most ? 1.f : exp2_fast(m - most),
                  [&](int c, const float(&x)[4]) { __builtin_memcpy(to + c, x, sizeof x); });
  }
  __syncthreads();
  for (int id = threadIdx.x; id < p.R * (DP / 4); id += 64 * W) {
    const int r = id / (DP / 4), c = id % (DP / 4) * 4;
    if (c >= p.D4) continue;
    float M = -INFINITY, sum = 0.f, rounded = 0.f, x[4] = {};
#pragma unroll
    for (int i = 0; i < W; ++i) M = fmaxf(M, stats[(i * 32 + r) * 3]);
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float *st = stats + (i * 32 + r) * 3, f = st[0] == M ? 1.f : exp2_fast(st[0] - M);
      sum = fmaf(st[1], f, sum), rounded = fmaf(st[2], f, rounded);
      const float4 v = *reinterpret_cast<const float4 *>(outs + ((size_t)i * p.R + r) * DP + c);
      x[0] += v.x, x[1] += v.y, x[2] += v.z, x[3] += v.w;
    }
    if (splits > 1) {
      float *to = part + (((int64_t)split * p.a.B * p.a.G + bg) * p.R + r) * (p.D4 + 4);
      __builtin_memcpy(to + c, x, sizeof x);
      if (c == 0) to[p.D4] = M, to[p.D4 + 1] = sum, to[p.D4 + 2] = rounded;
    } else {
      store_row_part<T>(p, g, b, (int64_t)bg * p.R + r, r, queries, c, x, M, sum, rounded);
    }
  }
}

}  // namespace

hipError_t launch_attention_few(const Attn &p, const Cut &c, float *part, hipStream_t s) {
  return by_dtype(p.a.dtype, [&](auto tag) {
    using T = decltype(tag);
    auto with = [&](auto dp, auto waves) {
      constexpr int DP = decltype(dp)::value, W = decltype(waves)::value;
      const size_t lds = few_lds<T, DP, W>(p.R);
      if (lds > 65536)
        if (hipError_t e = allow_lds<k_attn_few<T, DP, W>>(few_lds<T, DP, W>(32))) return e;
      return timed_launch("attn_few", k_attn_few<T, DP, W>, dim3((unsigned)(p.a.B * p.a.G * c.splits)), dim3(64 * W), lds, s, p,
                          part, c.splits, c.run, (int)(lds - (size_t)3 * W * 32 * sizeof(float)));
    };
    using std::integral_constant;
    if (p.a.D <= 32) return with(integral_constant<int, 32>{}, integral_constant<int, few_waves<T>(32)>{});
    if (p.a.D <= 64) return with(integral_constant<int, 64>{}, integral_constant<int, few_waves<T>(64)>{});
    if (p.a.D <= 96) return with(integral_constant<int, 96>{}, integral_constant<int, few_waves<T>(96)>{});
    return with(integral_constant<int, 128>{}, integral_constant<int, few_waves<T>(128)>{});
  });
}

}  // namespace fdc
