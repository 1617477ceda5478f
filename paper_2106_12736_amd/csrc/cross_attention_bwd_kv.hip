// Cross attention: the gradients of the keys and values.
#include "cross_attention.h"

namespace fdc {

using namespace attention;

namespace {

// gk and gv: a workgroup has 32 W keys and goes through a run of the rows (of every query head that shares them),
// whose q and gy pass through LDS.  k, v and both sums are in registers: 192 of a wave's for 16-bit keys of 128 channels, so that
// it has a SIMD to itself; the blocks of a tile are independent up to the sums, and the scores of one are formed
// among the products of another.  Four products: 8 x 2048 tokens over 1024 keys, 16 heads of 128 bf16, 390 to 412 us between
// runs (690 TFLOP/s), over 4096 keys 1435 (790 for what is added).  Bound by one wave's own latencies: with the blocks one after
// another 463 us, with both blocks' scores first 434, with the vector work set among the products 392.  Tried: v in LDS and
// eight waves of 256 registers (180 spilled); a branch around tiles without live rows, which has every sum copied
// between the two kinds of registers in each tile (253 moves for 64 products).  Registers spilled: float16's heads of 128 81
// (172 in workgroups of two waves), of 96 in two waves 36, bf16's of 128 in two waves 40; heads of 64 in eight waves bf16 18,
// float16 33.
// An order for COUNT products and the vector work that they are independent of: some instructions after each product, which
// the matrix unit takes 32 cycles for.
template <class T, int COUNT>
__device__ __forceinline__ void between() {
  if constexpr (std::is_same_v<T, __bf16>) {  // float16's scaling branches
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a product
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);  // reads from LDS
      __builtin_amdgcn_sched_group_barrier(0x402, 6, 0);  // vector instructions
    }
  }
}

// Whether one of row l % 32's values is NaN or an infinity: its exponent's bits, all set, carry into the sign's place.
template <class T, int N>
__device__ __forceinline__ bool odd_row(const Frag<T> (&x)[N]) {
  constexpr unsigned exponent = sizeof(T) == 4 ? 0x7f800000u : std::is_same_v<T, _Float16> ? 0x7c007c00u : 0x7f807f80u;
  constexpr unsigned one = sizeof(T) == 4 ? 0x00800000u : std::is_same_v<T, _Float16> ? 0x04000400u : 0x00800080u;
  constexpr int words = sizeof(Frag<T>) / 4;
  typedef unsigned Words __attribute__((ext_vector_type(words)));
  unsigned carry = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const Words w = __builtin_bit_cast(Words, x[i]);
#pragma unroll
    for (int j = 0; j < words; ++j) carry |= (w[j] & exponent) + one;
  }
  const uint64_t lanes = __ballot((carry & (sizeof(T) == 4 ? 0x80000000u : 0x80008000u)) != 0);
  return (lanes | lanes >> 32 | lanes << 32) >> (threadIdx.x & 63) & 1;
}

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
  float *lst = reinterpret_cast<float *>(lds_ + tiles_bytes<T, DP, W>());  // the rows' stats [2][QT], two buffers
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
  WaveRows<T, DP> wk, wv;
  wk.issue(static_cast<const T *>(p.a.k.p), offset_of(p.a.k, b, in, g), p.a.D, p.wide, there, lane);
  wv.issue(static_cast<const T *>(p.a.v.p), offset_of(p.a.v, b, in, g), p.a.D, p.wide, there, lane);
  v16f ok[DP / 32] = {}, ov[DP / 32] = {};
  Scaled<T> scaled;
  bool has_gk = there, has_gv = there;  // else they are 0
  uint64_t seen = 0;                    // whether there are rows
  const int first = split * run, last = min(first + run, (p.R + QT - 1) / QT);
  const float2 *rows = stats + (int64_t)bg * p.R;
  const float2 none{INFINITY, 0.f};
  if (first < last && __syncthreads_or(there)) {
    // 16-bit heads of 33 to 64 channels have no registers left for pieces that move (8 x 2048 rows on 1024 keys, 16 heads of 64
    // bf16 177 us, with them 192; of 63 channels, read by elements, 261, and 208 with them; float16 230 and 230, 300 and 256)
    using Tile = Staged<T, DP, 64 * W, !(DP == 64 && sizeof(T) == 2)>;
    Tile sq, sg;
    // where the pieces' rows are: a tile further on, as long as that is within the head
    constexpr int N = Tile::N;
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
      auto q_row = [&](int i) { return static_cast<const T *>(p.a.q.p) + q_at[i]; };
      auto g_row = [&](int i) { return static_cast<const T *>(gy.p) + g_at[i]; };
      // one branch for both: with one each, registers that the first loads were on their way to held addresses of the second,
      // which then waited for them (431 us in place of 390).  Heads of over 64 channels are more than a piece.
      if (DP > 64 || Tile::in_whole(p.a.D, p.wide))
        sq.load_whole(q_row, p.a.D), sg.load_whole(g_row, p.a.D);
      else
        sq.load_parts(q_row, p.a.D, live), sg.load_parts(g_row, p.a.D, live);
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
    wk.land(k, area, p.a.D, there, lane);
    wv.land(v, area, p.a.D, there, lane);
    __syncthreads();
    sq.store(lds, p.a.D, live), sg.store(lds + S, p.a.D, live);
    if (wave == 0 && lane < QT) lst[lane] = st.x, lst[QT + lane] = st.y;
    // The product of a key that holds NaN or an infinity with the zeros in the place of a row that is not there is NaN.  With a
    // row that is there its score is -inf, which adds nothing but what is NaN of delta (to gk), or has made the row's lse
    // NaN, and with it all.  So what is 0 is known here: the loop has no registers for it (scores that begin at -inf there: 436
    // us in place of 393 of the case above), and after it the lookup has the loop spill (float16's heads of 64: 204 in place of 126).
    const bool odd = odd_row<T>(k);
    if (__any(odd)) {
      bool no_lse = false, no_delta = false;
      for (int r = first * QT + lane; r < min(last * QT, p.R); r += 64) {
        no_lse |= rows[r].x != rows[r].x;
        no_delta |= !(fabsf(rows[r].y) < INFINITY);
      }
      no_lse = __any(no_lse), no_delta = __any(no_delta);
      if (odd) has_gv = no_lse, has_gk = no_lse || no_delta;
    }
    for (int tile = first; tile < last; ++tile) {
      const int buf = tile - first & 1;
      const T *qt = lds + buf * 2 * S, *gt = qt + S;
      const float *stt = lst + buf * 2 * QT;
      __syncthreads();
      const bool more = tile + 1 < last;
      const uint64_t live_next = __ballot(next.x != INFINITY);
      seen |= live;
      float2 after = none;
      if (more) {
        advance(tile + 1);
        load(live_next);
        after = stats_of(tile + 2);
      }
      {
        // The vector work of a block (probabilities, gradients of scores) stands among the products of its neighbours: block 0's
        // among block 1's scores, block 1's among block 0's sums.
        v16f s[NB], e[NB];
        Rows<T, DP, NS> rq[NB], rg[NB];
        Columns<T, DP> cg, cq;
        float4 lse[4], delta[4];
        auto read = [&](int q) { rq[q].load(qt, 32 * q, 0, lane), rg[q].load(gt, 32 * q, 0, lane); };
        auto read_stats = [&](int q) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            lse[i] = *reinterpret_cast<const float4 *>(stt + 32 * q + 8 * i + 4 * half);
            delta[i] = *reinterpret_cast<const float4 *>(stt + QT + 32 * q + 8 * i + 4 * half);
          }
        };
        auto scores = [&](int q) {
          s[q] = v16f{}, e[q] = v16f{};
#pragma unroll
          for (int i = 0; i < NS; ++i) {
            mma(s[q], rq[q].f[i], k[i]);
            mma(e[q], rg[q].f[i], v[i]);
          }
        };
        auto gradients = [&](int q) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float w[4] = {lse[i].x, lse[i].y, lse[i].z, lse[i].w}, y[4] = {delta[i].x, delta[i].y, delta[i].z, delta[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              s[q][4 * i + j] = exp2_fast(fmaf(s[q][4 * i + j], p.c, -w[j]));
              e[q][4 * i + j] = s[q][4 * i + j] * (e[q][4 * i + j] - y[j]);
            }
          }
        };
        read(0);
        read_stats(0);
        ahead<T>();
        if constexpr (NB > 1) read(NB - 1);
        scores(0);
        ahead<T>();
        cg.load(gt, 0, lane);
        if constexpr (NB > 1) scores(NB - 1);
        gradients(0);
        if constexpr (NB > 1) between<T, 2 * NS>();
        ahead<T>();
#pragma unroll
        for (int q = 0; q < NB; ++q) {
          cq.load(qt, 32 * q, lane);
          if (q + 1 < NB) read_stats(q + 1);
          cg.add_to(ov, {score_frag<T>(s[q], 0), score_frag<T>(s[q], 1)});
          if (q + 1 < NB) cg.load(gt, 32 * (q + 1), lane);
          scaled.fit(e[q], ok);
          cq.add_to(ok, {score_frag<T>(e[q], 0), score_frag<T>(e[q], 1)});
          if (q + 1 < NB) {
            gradients(q + 1);
            between<T, DP / 8>();
            ahead<T>();
          }
        }
      }
      if (more) {
        T *to = lds + (buf ^ 1) * 2 * S;
        sq.store(to, p.a.D, live_next), sg.store(to + S, p.a.D, live_next);
        if (wave == 0 && lane < QT) {
          float *to_stats = lst + (buf ^ 1) * 2 * QT + lane;
          to_stats[0] = next.x, to_stats[QT] = next.y;
        }
      }
      live = live_next, next = after;
    }
  }
  // whatever zeros in the place of the key, or of the rows, have led to
  if (!has_gk || seen == 0) {
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) ok[d] = v16f{};
  }
  if (!has_gv || seen == 0) {
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) ov[d] = v16f{};
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
  return by_shape<false>(p.a.dtype, p.a.D, c.waves, [&](auto tag, auto dp, auto waves) {
    using T = decltype(tag);
    constexpr int DP = decltype(dp)::value, W = decltype(waves)::value;
    return launch_tiles<k_attn_bwd_kv<T, DP, W>>("attn_bwd_kv", (long long)p.a.B * p.a.G * c.tiles * c.splits, 64 * W,
                                                 bwd_kv_lds<T, DP, W>(), s, p, gy, gk, gv, stats, part, c.tiles, c.splits,
                                                 c.run);
  });
}

}  // namespace fdc
