// Cross attention: the gradients of the keys and values.
#include "cross_attention.h"

namespace fdc {

using namespace attention;

namespace {

// gk and gv: a workgroup has 32 W keys and goes through a run of the rows (of every query head that shares them),
// whose q and gy pass through LDS.  k, v and both sums are in registers: 192 of a wave's for 16-bit keys of 128 channels, so that
// it has a SIMD to itself; the blocks of a tile are independent up to the sums, and the scores of one are formed
// among the products of another.
template <class T, int DP, int W>
constexpr size_t bwd_kv_lds() {
  return tiles_bytes<T, DP, W>() + 2 * attn_keys(sizeof(T)) * sizeof(float2);
}
template <class T, int DP, int W>
__global__ __launch_bounds__(64 * W, W / 4) void k_attn_bwd_kv(
    Attn p, fdc_heads gy, fdc_heads gk, fdc_heads gv, const float2 *__restrict__ stats, float *__restrict__ part,
    int key_tiles, int splits, int run) {
  constexpr int QT = attn_keys(sizeof(T)), S = QT * kStride<T, DP>, NB = QT / 32, NS = DP / 16;
  extern __shared__ __align__(16) char lds_[];
  T *lds = reinterpret_cast<T *>(lds_);
  float2 *lst = reinterpret_cast<float2 *>(lds_ + tiles_bytes<T, DP, W>());  // the rows' stats, two buffers
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  int id = xcd_remap(blockIdx.x, gridDim.x);
  const int kt = id % key_tiles;
  id /= key_tiles;
  const int split = id % splits, bg = id / splits, b = bg / p.a.G, g = bg - b * p.a.G;
  const int keys = length_of(p.a.lengths, b, p.a.Lk);
  const int key = (kt * W + wave) * 32 + (lane & 31);
  const bool there = key < keys && (p.a.mask == nullptr || p.a.mask[b * p.a.mask_stride + key] != 0);
  Frag<T> k[NS], v[NS];
  const int in = min(key, p.a.Lk - 1);
  T *area = lds + wave * 32 * kStride<T, DP>;
  WaveRows<T, DP>::load(k, area, static_cast<const T *>(p.a.k.p), offset_of(p.a.k, b, in, g), p.a.D, p.whole, there, lane);
  WaveRows<T, DP>::load(v, area, static_cast<const T *>(p.a.v.p), offset_of(p.a.v, b, in, g), p.a.D, p.whole, there, lane);
  __syncthreads();
  v16f ok[DP / 32] = {}, ov[DP / 32] = {};
  Scaled<T> scaled;
  const int first = split * run, last = min(first + run, (p.R + QT - 1) / QT);
  const float2 *rows = stats + (int64_t)bg * p.R;
  const float2 none{INFINITY, 0.f};
  if (first < last && __syncthreads_or(there)) {
    Staged<T, DP, 64 * W> sq, sg;
    // where the pieces' rows are: a tile further on, as long as that is within the head
    constexpr int N = Staged<T, DP, 64 * W>::N;
    int token[N];
    int64_t q_at[N], g_at[N];
    auto locate = [&](int i, int r) {
      const Row row = row_of(p, g, r, 0);
      token[i] = row.t;
      q_at[i] = offset_of(p.a.q, b, row.t, row.head), g_at[i] = offset_of(gy, b, row.t, row.head);
    };
#pragma unroll
    for (int i = 0; i < N; ++i) locate(i, first * QT + sq.row_of(i));
    auto load = [&](uint64_t live) {
      sq.load([&](int i) { return static_cast<const T *>(p.a.q.p) + q_at[i]; }, p.a.D, p.whole, live);
      sg.load([&](int i) { return static_cast<const T *>(gy.p) + g_at[i]; }, p.a.D, p.whole, live);
    };
    auto advance = [&](int tile) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        token[i] += QT;
        q_at[i] += QT * p.a.q.token_stride, g_at[i] += QT * gy.token_stride;
        if (token[i] >= p.a.Lq) locate(i, tile * QT + sq.row_of(i));
      }
    };
    auto stats_of = [&](int tile) {
      const int r = tile * QT + lane;
      return lane < QT && r < p.R ? rows[r] : none;
    };
    float2 st = stats_of(first), next = stats_of(first + 1);
    uint64_t live = __ballot(st.x != INFINITY);
    load(live);
    sq.store(lds, p.a.D, live), sg.store(lds + S, p.a.D, live);
    if (wave == 0 && lane < QT) lst[lane] = st;
    for (int tile = first; tile < last; ++tile) {
      const int buf = tile - first & 1;
      const T *qt = lds + buf * 2 * S, *gt = qt + S;
      const float2 *stt = lst + buf * QT;
      __syncthreads();
      const bool more = tile + 1 < last;
      const uint64_t live_next = __ballot(next.x != INFINITY);
      float2 after = none;
      if (more) {
        advance(tile + 1);
        load(live_next);
        after = stats_of(tile + 2);
      }
      {
#pragma unroll
        for (int q = 0; q < NB; ++q) {
          v16f s = {}, e = {};
          constexpr int H = NS / 2;
          Rows<T, DP, H> r0, r1;
          r0.load(qt, 32 * q, 0, lane);
          r1.load(qt, 32 * q, H, lane);
          ahead<T>();
#pragma unroll
          for (int i = 0; i < H; ++i) mma(s, r0.f[i], k[i]);
          r0.load(gt, 32 * q, 0, lane);
          ahead<T>();
#pragma unroll
          for (int i = 0; i < H; ++i) mma(s, r1.f[i], k[H + i]);
          r1.load(gt, 32 * q, H, lane);
          ahead<T>();
#pragma unroll
          for (int i = 0; i < H; ++i) mma(e, r0.f[i], v[i]);
          Columns<T, DP> cols;
          cols.load(gt, 32 * q, lane);
          ahead<T>();
#pragma unroll
          for (int i = 0; i < H; ++i) mma(e, r1.f[i], v[H + i]);
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const float2 w = stt[32 * q + 8 * (j / 4) + 4 * half + j % 4];
            s[j] = exp2_fast(fmaf(s[j], p.c, -w.x));
            e[j] = s[j] * (e[j] - w.y);
          }
          cols.add_to(ov, {score_frag<T>(s, 0), score_frag<T>(s, 1)});
          cols.load(qt, 32 * q, lane);
          scaled.fit(e, ok);
          cols.add_to(ok, {score_frag<T>(e, 0), score_frag<T>(e, 1)});
        }
      }
      if (more) {
        T *to = lds + (buf ^ 1) * 2 * S;
        sq.store(to, p.a.D, live_next), sg.store(to + S, p.a.D, live_next);
        if (wave == 0 && lane < QT) lst[(buf ^ 1) * QT + lane] = next;
      }
      live = live_next, next = after;
    }
  }
  if (!there) {  // whatever its zeros for k and v have led to
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) ok[d] = ov[d] = v16f{};
  }
  const float fv = exp2f(-kUpBack<T>), fk = p.a.scale * fv * scaled.undo();
  if (splits > 1) {
    if (key >= p.a.Lk) return;
    float *to = part + (((int64_t)split * p.a.B * p.a.G + bg) * p.a.Lk + key) * 2 * p.D4;
    each_four<DP>(ok, p.D4, half, fk, [&](int c, const float(&x)[4]) { __builtin_memcpy(to + c, x, sizeof x); });
    each_four<DP>(ov, p.D4, half, fv, [&](int c, const float(&x)[4]) { __builtin_memcpy(to + p.D4 + c, x, sizeof x); });
    return;
  }
  __syncthreads();
  WaveRows<T, DP>::store(area, static_cast<T *>(gk.p), offset_of(gk, b, in, g), p.a.D, key < p.a.Lk, lane,
                         [&](int d, int j) { return four<DP>(ok, d, j, fk); });
  WaveRows<T, DP>::store(area, static_cast<T *>(gv.p), offset_of(gv, b, in, g), p.a.D, key < p.a.Lk, lane,
                         [&](int d, int j) { return four<DP>(ov, d, j, fv); });
}

}  // namespace

hipError_t launch_attention_bwd_kv(const Attn &p, const Cut &c, const fdc_heads &gy, const fdc_heads &gk,
                                   const fdc_heads &gv, const float2 *stats, float *part, hipStream_t s) {
  return by_shape(p.a.dtype, p.a.D, c.waves, [&](auto tag, auto dp, auto waves) {
    using T = decltype(tag);
    constexpr int DP = decltype(dp)::value, W = decltype(waves)::value;
    return launch_tiles<k_attn_bwd_kv<T, DP, W>>("attn_bwd_kv", (long long)p.a.B * p.a.G * c.tiles * c.splits, 64 * W,
                                                 bwd_kv_lds<T, DP, W>(), s, p, gy, gk, gv, stats, part, c.tiles, c.splits,
                                                 c.run);
  });
}

}  // namespace fdc
