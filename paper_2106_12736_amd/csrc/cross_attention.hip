// Attention of tokens to states of another length: the forward, and what the backward's parts share.
#include "cross_attention.h"

namespace fdc {

using namespace attention;

namespace {

// ---- forward -----------------------------------------------------------------
// A workgroup has 32 W rows of a key head, a wave 32 of them, and goes through a run of the keys, whose
// tiles of k and v pass through LDS in two buffers: the next tile is loaded to registers during a tile's products.
// y is divided by the sum of the rounded probabilities, so that its weights add up to 1: for a row that reads one key
// almost alone, y then is off by a rounding of the others' part only, and so is delta.  lse is of the sum before rounding.
// Bound by the matrix units and what stands between their products: 8 x 2048 tokens over 1024 keys, 16 heads of 128 bf16,
// 187 to 194 us between runs (720 TFLOP/s), of which some 45 are rows in and out (201 MB, workgroups in step); over 4096 keys
// 658 us, 890 TFLOP/s for what is added, where a large library product runs at 1120.  Eight waves a workgroup share a tile's way through
// LDS (128 bytes a cycle feed the matrix units just in time).  Tried: tiles of 32 keys in workgroups of four waves, two on a
// compute unit (221 us).
// The running maximum of a row is raised, and its sums rescaled, only when a score is 2^8 past it.
template <class T, int DP, int W>
__global__ __launch_bounds__(64 * W, W / 4) void k_attn_fwd(Attn p, float *__restrict__ part, int row_tiles, int splits,
                                                     int run) {
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
  Frag<T> q[DP / 16];
  T *area = lds + wave * 32 * kStride<T, DP>;
  WaveRows<T, DP> wq;
  wq.issue(static_cast<const T *>(p.a.q.p), offset_of(p.a.q, b, row.t, row.head), p.a.D, p.wide, row.live, lane);
  v16f o[DP / 32] = {};
  float m = -INFINITY, l = 0.f, w = 0.f;  // the sum, and that of the rounded probabilities
  const int first = split * run, last = min(first + run, (keys + KT - 1) / KT);
  if (first < last && __syncthreads_or(row.live)) {
    Staged<T, DP, 64 * W> sk, sv;
    auto load = [&](int tile, uint64_t there) {
      const T *k0 = at<T>(p.a.k, b, (int64_t)tile * KT, g), *v0 = at<T>(p.a.v, b, (int64_t)tile * KT, g);
      const int most = p.a.Lk - 1 - tile * KT;
      sk.load([&](int i) { return k0 + min(sk.row_of(i), most) * p.a.k.token_stride; }, p.a.D, p.wide, there);
      sv.load([&](int i) { return v0 + min(sv.row_of(i), most) * p.a.v.token_stride; }, p.a.D, p.wide, there);
    };
    uint64_t there = keys_there(p, b, first * KT, keys, lane, KT), next = keys_there(p, b, (first + 1) * KT, keys, lane, KT);
    load(first, there);
    wq.land(q, area, p.a.D, row.live, lane);
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
        v16f s[NB] = {};
        Rows<T, DP, DP / 16> rows[NB];
#pragma unroll
        for (int k = 0; k < NB; ++k) rows[k].load(kt, 32 * k, 0, lane);
        ahead<T>();
#pragma unroll
        for (int k = 0; k < NB; ++k)
#pragma unroll
          for (int i = 0; i < DP / 16; ++i) mma(s[k], rows[k].f[i], q[i]);
        Columns<T, DP> cols;
        cols.load(vt, 0, lane);
        ahead<T>();
        if (there != (KT == 64 ? ~0ull : (1ull << KT) - 1)) {
          const uint64_t mine = there >> (4 * half);
#pragma unroll
          for (int k = 0; k < NB; ++k)
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (!(mine >> (32 * k + 8 * (j / 4) + j % 4) & 1)) s[k][j] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int k = 0; k < NB; ++k)
#pragma unroll
          for (int j = 0; j < 16; ++j) top = fmaxf(top, s[k][j]);
        top = halves_max(top) * p.c;
        const bool late = top > m + kLate;
        if (__any(late)) {
          const float to = late ? top : m, f = m == to ? 1.f : exp2_fast(m - to);
          l *= f, w *= f;
#pragma unroll
          for (int d = 0; d < DP / 32; ++d) o[d] *= f;
          m = to;
        }
        // a row whose scores are all -inf so far: its terms are 0
        const float base = kUp<T> - (m == -INFINITY ? 0.f : m);
#pragma unroll
        for (int k = 0; k < NB; ++k) {
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            s[k][j] = exp2_fast(fmaf(s[k][j], p.c, base));
            l += s[k][j];
          }
          const Frag<T> e[2] = {score_frag<T>(s[k], 0), score_frag<T>(s[k], 1)};
          if constexpr (sizeof(T) == 2) w = add_values(e[1], add_values(e[0], w));
          cols.add_to(o, e);
          if (k + 1 < NB) cols.load(vt, 32 * (k + 1), lane);
        }
      }
      if (more) {
        T *to = lds + (tile + 1 - first & 1) * 2 * S;
        sk.store(to, p.a.D, next), sv.store(to + S, p.a.D, next);
      }
      there = next, next = after;
    }
  }
  l = halves_sum(l);
  w = sizeof(T) == 2 ? halves_sum(w) : l;
  if (splits > 1) {
    if (r >= p.R) return;
    const int64_t at = ((int64_t)split * p.a.B * p.a.G + bg) * p.R + r;
    float *to = part + at * (p.D4 + 4);
    each_four<DP>(o, p.D4, half, 1.f, [&](int c, const float(&x)[4]) { __builtin_memcpy(to + c, x, sizeof x); });
    if (half == 0) to[p.D4] = m, to[p.D4 + 1] = l, to[p.D4 + 2] = w;
    return;
  }
  const bool none = !row.live || l == 0.f;
  const float f = none ? 0.f : 1.f / w;
  if (none) {  // not by a product: they are NaN where a key that the sequence has is, or infinite
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) o[d] = v16f{};
  }
  const int64_t at_row = (int64_t)bg * p.R + r;
  __syncthreads();
  WaveRows<T, DP>::store(area, static_cast<T *>(p.a.y.p), offset_of(p.a.y, b, row.t, row.head), p.a.D, r < p.R, lane,
                         [&](int d, int j) { return four<DP>(o, d, j, f); });
  if constexpr (sizeof(T) == 2) {
    if (p.low != nullptr)
      WaveRows<T, DP>::store(area, static_cast<T *>(p.low), at_row * p.D4, p.a.D, r < p.R, lane, [&](int d, int j) {
        const float4 x = four<DP>(o, d, j, f);
        return float4{low_of<T>(x.x), low_of<T>(x.y), low_of<T>(x.z), low_of<T>(x.w)};
      });
  }
  if (p.lse != nullptr && half == 0 && r < p.R)
    p.lse[at_row] = none ? -INFINITY : (m + __builtin_amdgcn_logf(l) - kUp<T>) * kLn2;
}

// The runs' results of a row, in order: a thread has 4 channels, and several runs' loads under way (HBM-bound; 42 runs of 1232
// rows of 96 channels 10 us, with one run's at a time 22).
template <class T>
__global__ __launch_bounds__(256) void k_attn_join(Attn p, const float *__restrict__ part, int splits,
                                                   long long total) {
  const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
  if (id >= total) return;
  const int fours = p.D4 / 4;
  const long long at_row = id / fours;
  const int c = (int)(id - at_row * fours) * 4;
  const int bg = (int)(at_row / p.R), b = bg / p.a.G, g = bg - b * p.a.G, r = (int)(at_row - (long long)bg * p.R);
  const int64_t step = (int64_t)p.a.B * p.a.G * p.R * (p.D4 + 4);
  const float *x = part + at_row * (p.D4 + 4);
  float m = -INFINITY, l = 0.f, w = 0.f, o[4] = {};
#pragma unroll 8
  for (int i = 0; i < splits; ++i) m = fmaxf(m, x[i * step + p.D4]);
#pragma unroll 8
  for (int i = 0; i < splits; ++i) {
    const float4 st = *reinterpret_cast<const float4 *>(x + i * step + p.D4), y = *reinterpret_cast<const float4 *>(x + i * step + c);
    const float f = st.x == m ? 1.f : exp2_fast(st.x - m);
    l = fmaf(st.y, f, l);
    w = fmaf(st.z, f, w);
    o[0] = fmaf(y.x, f, o[0]), o[1] = fmaf(y.y, f, o[1]), o[2] = fmaf(y.z, f, o[2]), o[3] = fmaf(y.w, f, o[3]);
  }
  store_row_part<T>(p, g, b, at_row, r, length_of(p.a.q_lengths, b, p.a.Lq), c, o, m, l, w);
}

// ---- backward ----------------------------------------------------------------
// Sums of the runs' parts [splits][B G][n][width D4], in order, to the heads of out0 and out1 (of the rows' tokens, or of
// the keys): a thread has 4 channels.
template <class T, bool Keys>
__global__ __launch_bounds__(256) void k_attn_sum(Attn p, const float *__restrict__ part, fdc_heads out0, fdc_heads out1,
                                                  int splits, int n, long long total) {
  const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
  if (id >= total) return;
  const int fours = p.D4 / 4 * (Keys ? 2 : 1);
  const long long at_row = id / fours;
  int c = (int)(id - at_row * fours) * 4;
  const int bg = (int)(at_row / n), b = bg / p.a.G, g = bg - b * p.a.G, r = (int)(at_row - (long long)bg * n);
  const float *x = part + at_row * (fours * 4) + c;
  float o[4] = {};
  const int64_t step = (int64_t)p.a.B * p.a.G * n * fours * 4;
#pragma unroll 8
  for (int i = 0; i < splits; ++i) {
    const float4 y = *reinterpret_cast<const float4 *>(x + i * step);
    o[0] += y.x, o[1] += y.y, o[2] += y.z, o[3] += y.w;
  }
  if constexpr (Keys) {
    const bool second = c >= p.D4;
    c -= second ? p.D4 : 0;
    store_some<T, 4>(at<T>(second ? out1 : out0, b, r, g) + c, o, p.a.D - c);
  } else {
    const Row row = row_of(p, g, r, 0);
    store_some<T, 4>(at<T>(out0, b, row.t, row.head) + c, o, p.a.D - c);
  }
}

}  // namespace

// The rows of a call, of any grouping: a thread for 4 channels where they are joined.
bool cross_attention_rows_fit(int64_t rows, int D) { return rows < 1LL << 36 && rows * ceil_div(D, 4) < (1LL << 32) - 256; }

// The largest number of workgroups of a launch: below 2^31, and below 2^32 threads.
bool cross_attention_fits(int dtype, int B, int Lq, int Lk, int H, int G, int D) {
  const Cuts c(dtype, B, Lq, Lk, H, G, D);
  const long long most = (1LL << 32) / 1024 - 1, heads = (long long)B * G;
  if (!cross_attention_rows_fit(c.rows, D) || c.keys >= 1LL << 36) return false;
  return heads * c.fwd.tiles * c.fwd.splits <= most && heads * c.kv.tiles * c.kv.splits <= most &&
         c.keys * 2 * c.D4 / 4 < (1LL << 32) - 256;
}

size_t cross_attention_saved(int dtype, int B, int Lq, int H, int D) {
  const size_t low = dtype_size(dtype) == 2 ? (size_t)B * Lq * H * (ceil_div(D, 4) * 4) * 2 : 0;
  return lse_floats(B, Lq, H) * sizeof(float) + (low + 15) / 16 * 16;
}
size_t cross_attention_fwd_ws(int dtype, int B, int Lq, int Lk, int H, int G, int D) {
  return Cuts(dtype, B, Lq, Lk, H, G, D).fwd_floats() * sizeof(float);
}
size_t cross_attention_bwd_ws(int dtype, int B, int Lq, int Lk, int H, int G, int D) {
  const Cuts c(dtype, B, Lq, Lk, H, G, D);
  return (c.stats_floats() + std::max(c.q_floats(), c.kv_floats())) * sizeof(float);
}

hipError_t launch_cross_attention_fwd(const fdc_cross_attention_args &a, float *saved, float *ws, hipStream_t s) {
  const Attn p = attn_of(a, saved);
  const Cuts cuts(a.dtype, a.B, a.Lq, a.Lk, a.H, a.G, a.D);
  const Cut &c = cuts.fwd;
  if (cuts.few) {
    if (hipError_t e = launch_attention_few(p, c, ws, s)) return e;
  } else if (hipError_t e = by_shape<true>(a.dtype, a.D, c.waves, [&](auto tag, auto dp, auto waves) {
        using T = decltype(tag);
        constexpr int DP = decltype(dp)::value, W = decltype(waves)::value;
        return launch_tiles<k_attn_fwd<T, DP, W>>("attn_fwd", (long long)a.B * a.G * c.tiles * c.splits, 64 * W,
                                                  tiles_bytes<T, DP, W>(), s, p, ws, c.tiles, c.splits, c.run);
             })) {
    return e;
  }
  if (c.splits == 1) return hipSuccess;
  const long long total = cuts.rows * (p.D4 / 4);
  return by_dtype(a.dtype, [&](auto tag) {
    return timed_launch("attn_join", k_attn_join<decltype(tag)>, dim3((unsigned)ceil_div(total, 256)), dim3(256), 0, s, p,
                        (const float *)ws, c.splits, total);
  });
}

hipError_t launch_cross_attention_bwd(const fdc_cross_attention_args &a, const float *saved,
                                      const fdc_cross_attention_grads &g, float *ws, hipStream_t s) {
  const Attn p = attn_of(a, const_cast<float *>(saved));
  const Cuts cuts(a.dtype, a.B, a.Lq, a.Lk, a.H, a.G, a.D);
  float2 *stats = reinterpret_cast<float2 *>(ws);
  float *part = ws + cuts.stats_floats();
  auto sum = [&](auto keys, const Cut &c, const fdc_heads &out0, const fdc_heads &out1, int n, long long total) {
    return by_dtype(a.dtype, [&](auto tag) {
      return timed_launch("attn_sum", k_attn_sum<decltype(tag), decltype(keys)::value>,
                          dim3((unsigned)ceil_div(total, 256)), dim3(256), 0, s, p, (const float *)part, out0, out1, c.splits,
                          n, total);
    });
  };
  const Cut &q = cuts.q, &kv = cuts.kv;
  if (hipError_t e = launch_attention_bwd_q(p, q, g.gy, g.gq, stats, part, s)) return e;
  if (q.splits > 1)
    if (hipError_t e = sum(std::false_type{}, q, g.gq, g.gq, p.R, cuts.rows * (p.D4 / 4))) return e;
  if (hipError_t e = launch_attention_bwd_kv(p, kv, g.gy, g.gk, g.gv, stats, part, s)) return e;
  if (kv.splits > 1) return sum(std::true_type{}, kv, g.gk, g.gv, a.Lk, cuts.keys * (2 * p.D4 / 4));
  return hipSuccess;
}

}  // namespace fdc
