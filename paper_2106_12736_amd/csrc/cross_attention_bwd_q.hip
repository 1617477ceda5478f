// Cross attention: the gradient of the queries.
#include "cross_attention.h"

namespace fdc {

using namespace attention;

namespace {

// A lane's channels of its row.
template <class T, int N>
__device__ __forceinline__ float dot(const Frag<T> (&x)[N], const Frag<T> (&y)[N]) {
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fmaf((float)x[i][e], (float)y[i][e], sum);
  return sum;
}

// gq: a workgroup has 32 W rows and goes through a run of the keys, as the forward does.  Before, its waves form their rows'
// delta from gy, y and y's low part, and the first run's leave it, with what a score's exponent is less by (infinity for a row
// without keys, or past the queries: its probabilities are 0), in stats [rows][2] for the gradient of k and v.  A launch of
// its own for these took 40 us of 8 x 2048 tokens, 16 heads of 128 bf16; here it takes 37, and 2 in place of 5 of small
// calls.  Three products: that case over 1024 keys 289 us, over 4096 keys 865 (1073 TFLOP/s for what is added, a large library
// product's 1120); the rest is rows in and out.  Half of a row's fragments are on their way from LDS at a time: all of them
// at once took the registers of two waves a SIMD (288 spilled; as it is 33 with 16-bit heads of 128 channels, 34 in
// float16, and 8 with those of 96; one is read back in a tile).
template <class T, int DP, int W>
__global__ __launch_bounds__(64 * W, W / 4) void k_attn_bwd_q(Attn p, fdc_heads gy, fdc_heads gq, float2 *__restrict__ stats,
                                                       float *__restrict__ part, int row_tiles, int splits, int run) {
  constexpr int KT = attn_keys(sizeof(T)), S = KT * kStride<T, DP>, NB = KT / 32;
  extern __shared__ __align__(16) char lds_[];
  T *lds = reinterpret_cast<T *>(lds_);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  int id = xcd_remap(blockIdx.x, gridDim.x);
  const int rt = id % row_tiles;
  id /= row_tiles;
  const int split = id % splits, bg = id / splits, b = bg / p.a.G, g = bg - b * p.a.G;
  const int keys = length_of(p.a.lengths, b, p.a.Lk), queries = length_of(p.a.q_lengths, b, p.a.Lq);
  const int r = (rt * W + wave) * 32 + (lane & 31);
  const Row row = row_of(p, g, r, queries);
  const int64_t at_row = (int64_t)bg * p.R + min(r, p.R - 1);
  const float lse = p.lse[at_row];
  const bool live = r < p.R && row.live && lse != -INFINITY;
  float2 st{live ? lse * kLog2e - kUpBack<T> : INFINITY, 0.f};
  Frag<T> q[DP / 16], go[DP / 16];
  T *area = lds + wave * 32 * kStride<T, DP>;
  WaveRows<T, DP> wq, wg, wy, wl;
  wq.issue(static_cast<const T *>(p.a.q.p), offset_of(p.a.q, b, row.t, row.head), p.a.D, p.wide, live, lane);
  wg.issue(static_cast<const T *>(gy.p), offset_of(gy, b, row.t, row.head), p.a.D, p.wide, live, lane);
  wy.issue(static_cast<const T *>(p.a.y.p), offset_of(p.a.y, b, row.t, row.head), p.a.D, p.wide, live, lane);
  if constexpr (sizeof(T) == 2) wl.issue(static_cast<const T *>(p.low), at_row * p.D4, p.a.D, p.wide, live, lane);
  v16f o[DP / 32] = {};
  Scaled<T> scaled;
  const int first = split * run, last = min(first + run, (keys + KT - 1) / KT);
  if (first < last && __syncthreads_or(live)) {
    Staged<T, DP, 64 * W> sk, sv;
    auto load = [&](int tile, uint64_t there) {
      const T *k0 = at<T>(p.a.k, b, (int64_t)tile * KT, g), *v0 = at<T>(p.a.v, b, (int64_t)tile * KT, g);
      const int most = p.a.Lk - 1 - tile * KT;
      sk.load([&](int i) { return k0 + min(sk.row_of(i), most) * p.a.k.token_stride; }, p.a.D, p.wide, there);
      sv.load([&](int i) { return v0 + min(sv.row_of(i), most) * p.a.v.token_stride; }, p.a.D, p.wide, there);
    };
    uint64_t there = keys_there(p, b, first * KT, keys, lane, KT), next = keys_there(p, b, (first + 1) * KT, keys, lane, KT);
    load(first, there);
    wq.land(q, area, p.a.D, live, lane);
    wg.land(go, area, p.a.D, live, lane);
    {
      Frag<T> y[DP / 16];
      wy.land(y, area, p.a.D, live, lane);
      st.y = dot<T>(go, y);
      if constexpr (sizeof(T) == 2) {
        wl.land(y, area, p.a.D, live, lane);
        st.y = fmaf(dot<T>(go, y), 1.f / kLowUp<T>, st.y);
      }
      st.y += __shfl_xor(st.y, 32, 64);
    }
    __syncthreads();
    sk.store(lds, p.a.D, there), sv.store(lds + S, p.a.D, there);
    for (int tile = first; tile < last; ++tile) {
      const T *kt = lds + (tile - first & 1) * 2 * S, *vt = kt + S;
      __syncthreads();
      const bool more = tile + 1 < last;
      uint64_t after = 0;
      if (more) {
        load(tile + 1, next);
        after = keys_there(p, b, (tile + 2) * KT, keys, lane, KT);
      }
      {
        const bool whole = there == (KT == 64 ? ~0ull : (1ull << KT) - 1);
        const uint64_t mine = there >> (4 * half);
#pragma unroll
        for (int k = 0; k < NB; ++k) {
          v16f s = {}, e = {};
          constexpr int H = DP / 32;  // half the steps: at most 32 registers on their way from LDS
          Rows<T, DP, H> r0, r1;
          r0.load(kt, 32 * k, 0, lane);
          r1.load(kt, 32 * k, H, lane);
          ahead<T>();
#pragma unroll
          for (int i = 0; i < H; ++i) mma(s, r0.f[i], q[i]);
          r0.load(vt, 32 * k, 0, lane);
          ahead<T>();
#pragma unroll
          for (int i = 0; i < H; ++i) mma(s, r1.f[i], q[H + i]);
          r1.load(vt, 32 * k, H, lane);
          ahead<T>();
#pragma unroll
          for (int i = 0; i < H; ++i) mma(e, r0.f[i], go[i]);
          Columns<T, DP> cols;
          cols.load(kt, 32 * k, lane);
          ahead<T>();
#pragma unroll
          for (int i = 0; i < H; ++i) mma(e, r1.f[i], go[H + i]);
#pragma unroll
          for (int j = 0; j < 16; ++j) s[j] = exp2_fast(fmaf(s[j], p.c, -st.x)) * (e[j] - st.y);
          if (!whole) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (!(mine >> (32 * k + 8 * (j / 4) + j % 4) & 1)) s[j] = 0.f;
          }
          scaled.fit(s, o);
          cols.add_to(o, {score_frag<T>(s, 0), score_frag<T>(s, 1)});
        }
      }
      if (more) {
        T *to = lds + (tile + 1 - first & 1) * 2 * S;
        sk.store(to, p.a.D, next), sv.store(to + S, p.a.D, next);
      }
      there = next, next = after;
    }
  }
  if (!live) {  // whatever NaN or infinities among the keys and values have led to
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) o[d] = v16f{};
  }
  if (split == 0 && half == 0 && r < p.R) stats[at_row] = st;
  const float f = p.a.scale * exp2f(-kUpBack<T>) * scaled.undo();
  if (splits > 1) {
    if (r >= p.R) return;
    float *to = part + (((int64_t)split * p.a.B * p.a.G + bg) * p.R + r) * p.D4;
    each_four<DP>(o, p.D4, half, f, [&](int c, const float(&x)[4]) { __builtin_memcpy(to + c, x, sizeof x); });
    return;
  }
  __syncthreads();
  WaveRows<T, DP>::store(area, static_cast<T *>(gq.p), offset_of(gq, b, row.t, row.head), p.a.D, r < p.R, lane,
                         [&](int d, int j) { return four<DP>(o, d, j, f); });
}

}  // namespace

hipError_t launch_attention_bwd_q(const Attn &p, const Cut &c, const fdc_heads &gy, const fdc_heads &gq,
                                  float2 *stats, float *part, hipStream_t s) {
  return by_shape<true>(p.a.dtype, p.a.D, c.waves, [&](auto tag, auto dp, auto waves) {
    using T = decltype(tag);
    constexpr int DP = decltype(dp)::value, W = decltype(waves)::value;
    return launch_tiles<k_attn_bwd_q<T, DP, W>>("attn_bwd_q", (long long)p.a.B * p.a.G * c.tiles * c.splits, 64 * W,
                                                tiles_bytes<T, DP, W>(), s, p, gy, gq, stats, part, c.tiles, c.splits, c.run);
  });
}

}  // namespace fdc
