// Attention of tokens to states of another length, forward and backward.
//
//   s = scale q k^T over the keys a sequence has,  p = exp(s - lse),  y = p v,  lse = log sum exp s
//   delta = gy . y,  gv = p^T gy,  gs = p (gy v^T - delta),  gq = scale gs k,  gk = scale gs^T q
//
// The rows of a key head g are those of the H / G query heads that share it, head by head: row r is token
// r % Lq of head g H / G + r / Lq, so that few tokens of many heads fill a tile too.
//
// Tiles are 32 x 32 products over 16 (v_mfma_f32_32x32x16 for 16-bit types, eight v_mfma_f32_32x32x2 for
// float32): lane l holds 8 values k = 8 (l / 32) + i of row (column) l % 32 of a factor, and of the
// result column l % 32, rows 8 (j / 4) + 4 (l / 32) + j % 4 in register j.  Scores are formed transposed, keys by
// queries, so that a lane has its query's statistics alone to hold, and its 8 registers 8 u ... of the scores are, without
// moving, the second factor of a product over the 16 keys 16 u + 8 (i / 4) + 4 (l / 32) + i % 4; the first
// factor's columns are read from LDS in that order (ds_read_b64_tr_b16 turns 4 x 16 pieces).
#include <algorithm>

#include "device.h"
#include "lds_limit.h"
#include "sequence.h"

namespace fdc {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef short v4s __attribute__((ext_vector_type(4)));

namespace {

// 8 values of a row for each lane.
template <class T>
struct Fragment {
  typedef T type __attribute__((ext_vector_type(8)));
};
template <class T>
using Frag = typename Fragment<T>::type;

__device__ __forceinline__ void mma(v16f &c, const Frag<__bf16> &a, const Frag<__bf16> &b) {
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ void mma(v16f &c, const Frag<_Float16> &a, const Frag<_Float16> &b) {
  c = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ void mma(v16f &c, const Frag<float> &a, const Frag<float> &b) {
#pragma unroll
  for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
}

// The values of the lanes l % 32 and l % 32 + 32, in both.
struct Halves {
  float lo, hi;
};
__device__ __forceinline__ Halves halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return {__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ float halves_max(float v) {
  const Halves h = halves(v);
  return fmaxf(h.lo, h.hi);
}
__device__ __forceinline__ float halves_sum(float v) {
  const Halves h = halves(v);
  return h.lo + h.hi;
}

constexpr int attn_keys(size_t size) { return size == 2 ? 64 : 32; }  // rows of an LDS tile
// A tile's rows are 32 bytes longer than their channels: 8 rows then begin at 8 different sets of 8 banks.
template <class T, int DP>
constexpr int kStride = DP + 32 / (int)sizeof(T);
template <class T, int DP>
constexpr size_t tile_bytes() {
  return (size_t)attn_keys(sizeof(T)) * kStride<T, DP> * sizeof(T);
}

// Row `row` of a tile, channels 16 s ... 16 s + 15 of which this lane's half.
template <class T, int DP>
__device__ __forceinline__ Frag<T> row_frag(const T *tile, int row, int s, int half) {
  return *reinterpret_cast<const Frag<T> *>(tile + row * kStride<T, DP> + 16 * s + 8 * half);
}
// Channel d0 + l % 32 of 16 rows of a tile from row0, in the order of the scores' registers.
template <class T, int DP>
__device__ __forceinline__ Frag<T> column_frag(const T *tile, int row0, int d0, int lane) {
  constexpr int S = kStride<T, DP>;
  const int half = lane >> 5;
  if constexpr (sizeof(T) == 2) {
    typedef __attribute__((address_space(3))) v4s *lds_t;
    const T *p = tile + (row0 + 4 * half + (lane & 15) / 4) * S + d0 + (lane & 16) + (lane & 3) * 4;
    struct {
      v4s lo, hi;
    } x{__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)p), __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(p + 8 * S))};
    return __builtin_bit_cast(Frag<T>, x);
  } else {
    const T *p = tile + (row0 + 4 * half) * S + d0 + (lane & 31);
    Frag<T> f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = p[(8 * (i / 4) + i % 4) * S];
    return f;
  }
}
// Registers 8 u ... 8 u + 7 of a tile of scores, rounded to the activations' type: at most half a step of each factor
// of a sum, as its other factors are.
template <class T>
__device__ __forceinline__ Frag<T> score_frag(const v16f &s, int u) {
  Frag<T> f;
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = (T)s[8 * u + i];
  return f;
}

// sum + the 8 values of a factor, added in float32.
__device__ __forceinline__ float add_values(const Frag<__bf16> &f, float sum) {
  typedef __bf16 v2 __attribute__((ext_vector_type(2)));
  const v2 one = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
  for (int i = 0; i < 8; i += 2) sum = __builtin_amdgcn_fdot2_f32_bf16(v2{f[i], f[i + 1]}, one, sum, false);
  return sum;
}
__device__ __forceinline__ float add_values(const Frag<_Float16> &f, float sum) {
  typedef _Float16 v2 __attribute__((ext_vector_type(2)));
  const v2 one = {(_Float16)1.f, (_Float16)1.f};
#pragma unroll
  for (int i = 0; i < 8; i += 2) sum = __builtin_amdgcn_fdot2(v2{f[i], f[i + 1]}, one, sum, false);
  return sum;
}

// n (maybe <= 0) of 8 elements from memory, the others 0.
template <class T>
__device__ __forceinline__ Frag<T> load_frag(const T *p, int n) {
  if (n >= 8) {
    Frag<T> f;
    __builtin_memcpy(&f, p, sizeof f);
    return f;
  }
  Frag<T> f{};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) f[i] = p[i];
  return f;
}
// The channels of a row of D as the factor of a product over channels.
template <class T, int DP>
__device__ __forceinline__ void load_row(Frag<T> (&f)[DP / 16], const T *p, int D, int half, bool there) {
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    f[s] = Frag<T>{};
    if (there) f[s] = load_frag<T>(p + 16 * s + 8 * half, D - 16 * s - 8 * half);
  }
}

// A tile on its way from memory to LDS, in 16-byte pieces of its rows; rows whose bit of `there` is not set are 0.
template <class T, int DP, int TH>
struct Staged {
  static constexpr int V = 16 / (int)sizeof(T), PR = DP / V, COUNT = attn_keys(sizeof(T)) * PR, N = (COUNT + TH - 1) / TH;
  Pack<T, V> x[N];
  // at(row): where row `row` of the tile begins
  template <class At>
  __device__ __forceinline__ void load(At &&at, int D, uint64_t there) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = (int)threadIdx.x + i * TH, row = id / PR, c = id % PR * V;
      x[i] = Pack<T, V>{};
      if ((COUNT % TH == 0 || id < COUNT) && c < D && (there >> row & 1)) x[i] = load_some<T, V>(at(row) + c, D - c);
    }
  }
  __device__ __forceinline__ void store(T *tile) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = (int)threadIdx.x + i * TH, row = id / PR, c = id % PR * V;
      if (COUNT % TH == 0 || id < COUNT) *reinterpret_cast<Pack<T, V> *>(tile + row * kStride<T, DP> + c) = x[i];
    }
  }
};

// What the kernels share of a call.
struct Attn {
  fdc_cross_attention_args a;
  int per, R;  // query heads a key head, rows a key head
  int D4;      // channels of a partial result's row
  float c;     // scale log2(e)
  float *lse;  // [B][H][Lq] (NULL: no backward follows)
  void *low;   // [rows][D4], 16-bit types: what y's rounding lost, times kLowUp
};
// y and its low part are the sum to 16 (bfloat16) or 22 (float16) bits: delta is formed from both, since for a row that reads
// few keys it nearly cancels against gy . v, and y's rounding alone would be the largest error of gq and gk.  The
// factor keeps the low part among float16's normal numbers where y is.
template <class T>
constexpr float kLowUp = std::is_same_v<T, _Float16> ? 2048.f : 1.f;

// Row r of key head g: a head and a token.
struct Row {
  int head, t;
  bool live;
};
__device__ __forceinline__ Row row_of(const Attn &p, int g, int r, int queries) {
  const int hh = r / p.a.Lq, t = r - hh * p.a.Lq;
  return {g * p.per + hh, t, r < p.R && t < queries};
}
template <class T>
__device__ __forceinline__ T *at(const fdc_heads &x, int b, int64_t t, int64_t h) {
  return static_cast<T *>(x.p) + b * x.batch_stride + t * x.token_stride + h * x.head_stride;
}

// Which of the 64 keys from key0 sequence b has, the same in every lane.
__device__ __forceinline__ uint64_t keys_there(const Attn &p, int b, int key0, int keys, int lane, int width) {
  const int key = key0 + lane;
  bool there = lane < width && key < keys;
  if (there && p.a.mask != nullptr) there = p.a.mask[b * p.a.mask_stride + key] != 0;
  return __ballot(there);
}

template <int DP, class F>
__device__ __forceinline__ void each_four(const v16f (&o)[DP / 32], int D, int half, float f, F &&store) {
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = 32 * d + 8 * j + 4 * half;
      const float x[4] = {o[d][4 * j] * f, o[d][4 * j + 1] * f, o[d][4 * j + 2] * f, o[d][4 * j + 3] * f};
      if (c < D) store(c, x);
    }
}

// 4 channels of a row of y from c on, and of its low part.
template <class T>
__device__ __forceinline__ void store_y(const Attn &p, T *y, int64_t at_row, int c, const float (&x)[4]) {
  store_some<T, 4>(y + c, x, p.a.D - c);
  if constexpr (sizeof(T) == 2) {
    if (p.low != nullptr) {
      float rest[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) rest[i] = (x[i] - (float)(T)x[i]) * kLowUp<T>;
      store_pack<T, 4>(static_cast<T *>(p.low) + at_row * p.D4 + c, rest);
    }
  }
}

// ---- forward -----------------------------------------------------------------
// float16's probabilities are held 2^7 times as large, so that small ones keep their digits (2^-14 is its least normal
// number); they stay below 2^15 with the largest score up to 2^8 past the one they are taken relative to.
template <class T>
constexpr float kUp = std::is_same_v<T, _Float16> ? 7.f : 0.f;
constexpr float kLate = 8.f;

// A workgroup has 32 W rows of a key head, a wave 32 of them, and goes through a run of the keys, whose
// tiles of k and v pass through LDS in two buffers: the next tile is loaded to registers during a tile's products.
// y is divided by the sum of the rounded probabilities, so that its weights add up to 1: for a row that reads one key
// almost alone, y then is off by a rounding of the others' part only, and so is delta.  lse is of the sum before rounding.
// The running maximum of a row is raised, and its sums rescaled, only when a score is 2^8 past it.
template <class T, int DP, int W>
__global__ __launch_bounds__(64 * W) void k_attn_fwd(Attn p, float *__restrict__ part, int row_tiles, int splits,
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
  load_row<T, DP>(q, at<T>(p.a.q, b, row.t, row.head), p.a.D, half, row.live);
  v16f o[DP / 32] = {};
  float m = -INFINITY, l = 0.f, w = 0.f;  // the sum, and that of the rounded probabilities
  const int first = split * run, last = min(first + run, (keys + KT - 1) / KT);
  if (first < last && __syncthreads_or(row.live)) {
    Staged<T, DP, 64 * W> sk, sv;
    auto load = [&](int tile, uint64_t there) {
      const T *k0 = at<T>(p.a.k, b, (int64_t)tile * KT, g), *v0 = at<T>(p.a.v, b, (int64_t)tile * KT, g);
      sk.load([&](int i) { return k0 + i * p.a.k.token_stride; }, p.a.D, there);
      sv.load([&](int i) { return v0 + i * p.a.v.token_stride; }, p.a.D, there);
    };
    uint64_t there = keys_there(p, b, first * KT, keys, lane, KT), next = keys_there(p, b, (first + 1) * KT, keys, lane, KT);
    load(first, there);
    sk.store(lds), sv.store(lds + S);
    for (int tile = first; tile < last; ++tile) {
      const T *kt = lds + (tile - first & 1) * 2 * S, *vt = kt + S;
      __syncthreads();
      const bool more = tile + 1 < last;
      uint64_t after = 0;
      if (more) {
        load(tile + 1, next);
        after = keys_there(p, b, (tile + 2) * KT, keys, lane, KT);
      }
      if (there != 0) {
        v16f s[NB] = {};
#pragma unroll
        for (int k = 0; k < NB; ++k)
#pragma unroll
          for (int i = 0; i < DP / 16; ++i) mma(s[k], row_frag<T, DP>(kt, 32 * k + (lane & 31), i, half), q[i]);
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
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const Frag<T> e = score_frag<T>(s[k], u);
            if constexpr (sizeof(T) == 2) w = add_values(e, w);
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) mma(o[d], column_frag<T, DP>(vt, 32 * k + 16 * u, 32 * d, lane), e);
          }
        }
      }
      if (more) {
        T *to = lds + (tile + 1 - first & 1) * 2 * S;
        sk.store(to), sv.store(to + S);
      }
      there = next, next = after;
    }
  }
  l = halves_sum(l);
  w = sizeof(T) == 2 ? halves_sum(w) : l;
  if (r >= p.R) return;
  if (splits > 1) {
    const int64_t at = ((int64_t)split * p.a.B * p.a.G + bg) * p.R + r;
    float *to = part + at * (p.D4 + 4);
    each_four<DP>(o, p.D4, half, 1.f, [&](int c, const float(&x)[4]) { __builtin_memcpy(to + c, x, sizeof x); });
    if (half == 0) to[p.D4] = m, to[p.D4 + 1] = l, to[p.D4 + 2] = w;
    return;
  }
  const float f = !row.live || l == 0.f ? 0.f : 1.f / w;
  T *y = at<T>(p.a.y, b, row.t, row.head);
  const int64_t at_row = (int64_t)bg * p.R + r;
  each_four<DP>(o, p.a.D, half, f, [&](int c, const float(&x)[4]) { store_y<T>(p, y, at_row, c, x); });
  if (p.lse != nullptr && half == 0)
    p.lse[at_row] = !row.live || l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l) - kUp<T>) * kLn2;
}

// The runs' results of a row, in order: a thread has 4 channels.
template <class T>
__global__ __launch_bounds__(256) void k_attn_join(Attn p, const float *__restrict__ part, int splits,
                                                   long long total) {
  const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
  if (id >= total) return;
  const int fours = p.D4 / 4;
  const long long at_row = id / fours;
  const int c = (int)(id - at_row * fours) * 4;
  const int bg = (int)(at_row / p.R), b = bg / p.a.G, g = bg - b * p.a.G;
  const Row row = row_of(p, g, (int)(at_row - (long long)bg * p.R), length_of(p.a.q_lengths, b, p.a.Lq));
  const int64_t step = (int64_t)p.a.B * p.a.G * p.R * (p.D4 + 4);
  const float *x = part + at_row * (p.D4 + 4);
  float m = -INFINITY, l = 0.f, w = 0.f, o[4] = {};
  for (int i = 0; i < splits; ++i) m = fmaxf(m, x[i * step + p.D4]);
  for (int i = 0; i < splits; ++i) {
    const float *y = x + i * step, f = y[p.D4] == m ? 1.f : exp2_fast(y[p.D4] - m);
    l = fmaf(y[p.D4 + 1], f, l);
    w = fmaf(y[p.D4 + 2], f, w);
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = fmaf(y[c + j], f, o[j]);
  }
  const float f = !row.live || l == 0.f ? 0.f : 1.f / w;
#pragma unroll
  for (int j = 0; j < 4; ++j) o[j] *= f;
  store_y<T>(p, at<T>(p.a.y, b, row.t, row.head), at_row, c, o);
  if (p.lse != nullptr && c == 0)
    p.lse[at_row] = !row.live || l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l) - kUp<T>) * kLn2;
}

// ---- backward ----------------------------------------------------------------
// float16's probabilities times 2^15 (at most 2^15): 2^-14 is its least normal number.
template <class T>
constexpr float kUpBack = std::is_same_v<T, _Float16> ? 15.f : 0.f;

// [rows][2]: what a score's exponent is less by (infinity for a row without keys, or past the queries: its probabilities are 0)
// and delta.  16 lanes a row.
template <class T>
__global__ __launch_bounds__(256) void k_attn_delta(Attn p, fdc_heads gy, float2 *__restrict__ stats,
                                                    long long rows) {
  const long long at_row = (long long)blockIdx.x * 16 + threadIdx.x / 16;
  if (at_row >= rows) return;
  const int bg = (int)(at_row / p.R), b = bg / p.a.G, g = bg - b * p.a.G, c = threadIdx.x % 16 * 8;
  const Row row = row_of(p, g, (int)(at_row - (long long)bg * p.R), length_of(p.a.q_lengths, b, p.a.Lq));
  const float e = p.lse[at_row];
  const bool live = row.live && e != -INFINITY;
  float sum = 0.f;
  if (live && c < p.a.D) {
    const Frag<T> x = load_frag<T>(at<T>(gy, b, row.t, row.head) + c, p.a.D - c);
    const Frag<T> y = load_frag<T>(at<T>(p.a.y, b, row.t, row.head) + c, p.a.D - c);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fmaf((float)x[i], (float)y[i], sum);
    if constexpr (sizeof(T) == 2) {
      const Frag<T> rest = load_frag<T>(static_cast<const T *>(p.low) + at_row * p.D4 + c, p.a.D - c);
      float more = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) more = fmaf((float)x[i], (float)rest[i], more);
      sum = fmaf(more, 1.f / kLowUp<T>, sum);
    }
  }
  sum = lane_sum<16>(sum);
  if (threadIdx.x % 16 == 0) stats[at_row] = live ? float2{e * kLog2e - kUpBack<T>, sum} : float2{INFINITY, 0.f};
}

// The gradients of scores as the factor of a product.  In float16 a column of them is scaled by a power of two
// of its own, chosen by its largest value so far, so that neither small gradients lose their digits nor large ones overflow;
// the sums made with them carry it.
template <class T>
struct Scaled {
  float f = 1.f;
  template <int N>
  __device__ __forceinline__ void fit(v16f &, v16f (&)[N]) {}
  __device__ __forceinline__ float undo() const { return 1.f; }
};
template <>
struct Scaled<_Float16> {
  float f = 0x1p100f;
  template <int N>
  __device__ __forceinline__ void fit(v16f &s, v16f (&sums)[N]) {
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) top = fmaxf(top, fabsf(s[j]));
    top = halves_max(top);
    if (__any(top * f > 32768.f)) {
      // to 2^10 ... 2^11: room for 16 times as large ones
      const float to = top * f > 32768.f ? ldexpf(1.f, 11 - __builtin_amdgcn_frexp_expf(top)) : f, by = to / f;
#pragma unroll
      for (int d = 0; d < N; ++d) sums[d] *= by;
      f = to;
    }
    s *= f;
  }
  __device__ __forceinline__ float undo() const { return 1.f / f; }
};

// gq: a workgroup has 32 W rows and goes through a run of the keys, as the forward does.
template <class T, int DP, int W>
__global__ __launch_bounds__(64 * W) void k_attn_bwd_q(Attn p, fdc_heads gy, fdc_heads gq, const float2 *__restrict__ stats,
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
  const float2 st = r < p.R ? stats[(int64_t)bg * p.R + r] : float2{INFINITY, 0.f};
  const bool live = st.x != INFINITY;
  Frag<T> q[DP / 16], go[DP / 16];
  load_row<T, DP>(q, at<T>(p.a.q, b, row.t, row.head), p.a.D, half, live);
  load_row<T, DP>(go, at<T>(gy, b, row.t, row.head), p.a.D, half, live);
  v16f o[DP / 32] = {};
  Scaled<T> scaled;
  const int first = split * run, last = min(first + run, (keys + KT - 1) / KT);
  if (first < last && __syncthreads_or(live)) {
    Staged<T, DP, 64 * W> sk, sv;
    auto load = [&](int tile, uint64_t there) {
      const T *k0 = at<T>(p.a.k, b, (int64_t)tile * KT, g), *v0 = at<T>(p.a.v, b, (int64_t)tile * KT, g);
      sk.load([&](int i) { return k0 + i * p.a.k.token_stride; }, p.a.D, there);
      sv.load([&](int i) { return v0 + i * p.a.v.token_stride; }, p.a.D, there);
    };
    uint64_t there = keys_there(p, b, first * KT, keys, lane, KT), next = keys_there(p, b, (first + 1) * KT, keys, lane, KT);
    load(first, there);
    sk.store(lds), sv.store(lds + S);
    for (int tile = first; tile < last; ++tile) {
      const T *kt = lds + (tile - first & 1) * 2 * S, *vt = kt + S;
      __syncthreads();
      const bool more = tile + 1 < last;
      uint64_t after = 0;
      if (more) {
        load(tile + 1, next);
        after = keys_there(p, b, (tile + 2) * KT, keys, lane, KT);
      }
      if (there != 0) {
        const bool whole = there == (KT == 64 ? ~0ull : (1ull << KT) - 1);
        const uint64_t mine = there >> (4 * half);
#pragma unroll
        for (int k = 0; k < NB; ++k) {
          v16f s = {}, e = {};
#pragma unroll
          for (int i = 0; i < DP / 16; ++i) mma(s, row_frag<T, DP>(kt, 32 * k + (lane & 31), i, half), q[i]);
#pragma unroll
          for (int i = 0; i < DP / 16; ++i) mma(e, row_frag<T, DP>(vt, 32 * k + (lane & 31), i, half), go[i]);
#pragma unroll
          for (int j = 0; j < 16; ++j) s[j] = exp2_fast(fmaf(s[j], p.c, -st.x)) * (e[j] - st.y);
          if (!whole) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (!(mine >> (32 * k + 8 * (j / 4) + j % 4) & 1)) s[j] = 0.f;
          }
          scaled.fit(s, o);
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const Frag<T> f = score_frag<T>(s, u);
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) mma(o[d], column_frag<T, DP>(kt, 32 * k + 16 * u, 32 * d, lane), f);
          }
        }
      }
      if (more) {
        T *to = lds + (tile + 1 - first & 1) * 2 * S;
        sk.store(to), sv.store(to + S);
      }
      there = next, next = after;
    }
  }
  if (r >= p.R) return;
  const float f = p.a.scale * exp2f(-kUpBack<T>) * scaled.undo();
  if (splits > 1) {
    float *to = part + (((int64_t)split * p.a.B * p.a.G + bg) * p.R + r) * p.D4;
    each_four<DP>(o, p.D4, half, f, [&](int c, const float(&x)[4]) { __builtin_memcpy(to + c, x, sizeof x); });
    return;
  }
  T *to = at<T>(gq, b, row.t, row.head);
  each_four<DP>(o, p.a.D, half, f, [&](int c, const float(&x)[4]) { store_some<T, 4>(to + c, x, p.a.D - c); });
}

// gk and gv: a workgroup has 32 W keys and goes through a run of the rows (of every query head that shares them),
// whose q and gy pass through LDS.
template <class T, int DP, int W>
__global__ __launch_bounds__(64 * W) void k_attn_bwd_kv(Attn p, fdc_heads gy, fdc_heads gk, fdc_heads gv,
                                                        const float2 *__restrict__ stats, float *__restrict__ part,
                                                        int key_tiles, int splits, int run) {
  constexpr int QT = attn_keys(sizeof(T)), S = QT * kStride<T, DP>;
  extern __shared__ __align__(16) char lds_[];
  T *lds = reinterpret_cast<T *>(lds_);
  float2 *lst = reinterpret_cast<float2 *>(lds + 4 * S);  // the rows' stats, two buffers
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  int id = xcd_remap(blockIdx.x, gridDim.x);
  const int kt = id % key_tiles;
  id /= key_tiles;
  const int split = id % splits, bg = id / splits, b = bg / p.a.G, g = bg - b * p.a.G;
  const int keys = length_of(p.a.lengths, b, p.a.Lk);
  const int key = (kt * W + wave) * 32 + (lane & 31);
  const bool there = key < keys && (p.a.mask == nullptr || p.a.mask[b * p.a.mask_stride + key] != 0);
  Frag<T> k[DP / 16], v[DP / 16];
  load_row<T, DP>(k, at<T>(p.a.k, b, key, g), p.a.D, half, there);
  load_row<T, DP>(v, at<T>(p.a.v, b, key, g), p.a.D, half, there);
  v16f ok[DP / 32] = {}, ov[DP / 32] = {};
  Scaled<T> scaled;
  const int first = split * run, last = min(first + run, (p.R + QT - 1) / QT);
  const float2 *rows = stats + (int64_t)bg * p.R;
  const float2 none{INFINITY, 0.f};
  if (first < last && __syncthreads_or(there)) {
    Staged<T, DP, 64 * W> sq, sg;
    auto load = [&](int tile, uint64_t live) {
      auto row_at = [&](const fdc_heads &x, int i) {
        const Row row = row_of(p, g, tile * QT + i, 0);
        return at<T>(x, b, row.t, row.head);
      };
      sq.load([&](int i) { return row_at(p.a.q, i); }, p.a.D, live);
      sg.load([&](int i) { return row_at(gy, i); }, p.a.D, live);
    };
    auto stats_of = [&](int tile) {
      const int r = tile * QT + lane;
      return lane < QT && r < p.R ? rows[r] : none;
    };
    float2 st = stats_of(first), next = stats_of(first + 1);
    uint64_t live = __ballot(st.x != INFINITY);
    load(first, live);
    sq.store(lds), sg.store(lds + S);
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
        load(tile + 1, live_next);
        after = stats_of(tile + 2);
      }
      if (live != 0) {
#pragma unroll
        for (int q = 0; q < QT / 32; ++q) {
          v16f s = {}, e = {};
#pragma unroll
          for (int i = 0; i < DP / 16; ++i) mma(s, row_frag<T, DP>(qt, 32 * q + (lane & 31), i, half), k[i]);
#pragma unroll
          for (int i = 0; i < DP / 16; ++i) mma(e, row_frag<T, DP>(gt, 32 * q + (lane & 31), i, half), v[i]);
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const float2 w = stt[32 * q + 8 * (j / 4) + 4 * half + j % 4];
            s[j] = exp2_fast(fmaf(s[j], p.c, -w.x));
            e[j] = s[j] * (e[j] - w.y);
          }
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const Frag<T> f = score_frag<T>(s, u);
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) mma(ov[d], column_frag<T, DP>(gt, 32 * q + 16 * u, 32 * d, lane), f);
          }
          scaled.fit(e, ok);
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const Frag<T> f = score_frag<T>(e, u);
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) mma(ok[d], column_frag<T, DP>(qt, 32 * q + 16 * u, 32 * d, lane), f);
          }
        }
      }
      if (more) {
        T *to = lds + (buf ^ 1) * 2 * S;
        sq.store(to), sg.store(to + S);
        if (wave == 0 && lane < QT) lst[(buf ^ 1) * QT + lane] = next;
      }
      live = live_next, next = after;
    }
  }
  if (key >= p.a.Lk) return;
  if (!there) {  // whatever its zeros for k and v have led to
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) ok[d] = ov[d] = v16f{};
  }
  const float fv = exp2f(-kUpBack<T>), fk = p.a.scale * fv * scaled.undo();
  if (splits > 1) {
    float *to = part + (((int64_t)split * p.a.B * p.a.G + bg) * p.a.Lk + key) * 2 * p.D4;
    each_four<DP>(ok, p.D4, half, fk, [&](int c, const float(&x)[4]) { __builtin_memcpy(to + c, x, sizeof x); });
    each_four<DP>(ov, p.D4, half, fv, [&](int c, const float(&x)[4]) { __builtin_memcpy(to + p.D4 + c, x, sizeof x); });
    return;
  }
  T *tk = at<T>(gk, b, key, g), *tv = at<T>(gv, b, key, g);
  each_four<DP>(ok, p.a.D, half, fk, [&](int c, const float(&x)[4]) { store_some<T, 4>(tk + c, x, p.a.D - c); });
  each_four<DP>(ov, p.a.D, half, fv, [&](int c, const float(&x)[4]) { store_some<T, 4>(tv + c, x, p.a.D - c); });
}

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
  for (int i = 0; i < splits; ++i) {
    const float *y = x + i * ((int64_t)p.a.B * p.a.G * n * fours * 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] += y[j];
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

// ---- host ----------------------------------------------------------------------
// Workgroups of `waves` waves that have 32 rows (or keys) each, and runs of the tiles they go through.
struct Cut {
  int waves, tiles, splits, run;
};
Cut cut(long long heads, long long own, long long through, int tile) {
  Cut c;
  c.waves = own > 128 && heads * ceil_div(own, 256) >= 256 ? 8 : own > 64 ? 4 : 2;
  c.tiles = (int)ceil_div(own, 32 * c.waves);
  const long long steps = ceil_div(through, tile), blocks = heads * c.tiles;
  const long long splits = std::max(1LL, std::min(ceil_div(512, blocks), steps / 2));
  c.run = (int)ceil_div(steps, splits);
  c.splits = (int)ceil_div(steps, c.run);
  return c;
}
struct Cuts {
  Cut fwd, q, kv;
  long long rows, keys, D4;
  Cuts(int dtype, int B, int Lq, int Lk, int H, int G, int D) {
    const long long heads = (long long)B * G, R = (long long)H / G * Lq;
    const int tile = attn_keys(dtype_size(dtype));
    fwd = q = cut(heads, R, Lk, tile);
    kv = cut(heads, Lk, R, tile);
    rows = heads * R, keys = heads * Lk, D4 = ceil_div(D, 4) * 4;
  }
  size_t fwd_floats() const { return fwd.splits > 1 ? (size_t)fwd.splits * rows * (D4 + 4) : 0; }
  size_t stats_floats() const { return (size_t)ceil_div(rows * 2, 4) * 4; }
  size_t q_floats() const { return q.splits > 1 ? (size_t)q.splits * rows * D4 : 0; }
  size_t kv_floats() const { return kv.splits > 1 ? (size_t)kv.splits * keys * 2 * D4 : 0; }
};

int64_t lse_floats(int B, int Lq, int H) { return ceil_div((int64_t)B * Lq * H, 4) * 4; }
Attn attn_of(const fdc_cross_attention_args &a, float *saved) {
  void *low = saved != nullptr && dtype_size(a.dtype) == 2 ? saved + lse_floats(a.B, a.Lq, a.H) : nullptr;
  return {a, a.H / a.G, a.H / a.G * a.Lq, (a.D + 3) / 4 * 4, a.scale * kLog2e, saved, low};
}

// f(T{}, padded channels, waves) for the type, channels and waves of a call.
template <class F>
hipError_t by_shape(int dtype, int D, int waves, F &&f) {
  using std::integral_constant;
  return by_dtype(dtype, [&](auto tag) {
    auto with = [&](auto dp) {
      if (waves == 8) return f(tag, dp, integral_constant<int, 8>{});
      if (waves == 4) return f(tag, dp, integral_constant<int, 4>{});
      return f(tag, dp, integral_constant<int, 2>{});
    };
    if (D <= 32) return with(integral_constant<int, 32>{});
    if (D <= 64) return with(integral_constant<int, 64>{});
    if (D <= 96) return with(integral_constant<int, 96>{});
    return with(integral_constant<int, 128>{});
  });
}
template <auto Kern, class... Args>
hipError_t launch_tiles(const char *name, long long blocks, int threads, size_t lds, hipStream_t s, Args... args) {
  if (lds > 65536)
    if (hipError_t e = allow_lds<Kern>(lds)) return e;
  return timed_launch(name, Kern, dim3((unsigned)blocks), dim3(threads), lds, s, args...);
}

}  // namespace

// The largest number of workgroups of a launch: below 2^31, and below 2^32 threads.
bool cross_attention_fits(int dtype, int B, int Lq, int Lk, int H, int G, int D) {
  const Cuts c(dtype, B, Lq, Lk, H, G, D);
  const long long most = (1LL << 32) / 512 - 1, heads = (long long)B * G;
  if (c.rows >= 1LL << 36 || c.keys >= 1LL << 36) return false;
  return heads * c.fwd.tiles * c.fwd.splits <= most && heads * c.kv.tiles * c.kv.splits <= most &&
         c.rows * c.D4 / 4 < (1LL << 32) - 256 && c.keys * 2 * c.D4 / 4 < (1LL << 32) - 256;
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
  if (hipError_t e = by_shape(a.dtype, a.D, c.waves, [&](auto tag, auto dp, auto waves) {
        using T = decltype(tag);
        constexpr int DP = decltype(dp)::value, W = decltype(waves)::value;
        return launch_tiles<k_attn_fwd<T, DP, W>>("attn_fwd", (long long)a.B * a.G * c.tiles * c.splits, 64 * W,
                                                  4 * tile_bytes<T, DP>(), s, p, ws, c.tiles, c.splits, c.run);
      }))
    return e;
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
  if (hipError_t e = by_dtype(a.dtype, [&](auto tag) {
        return timed_launch("attn_delta", k_attn_delta<decltype(tag)>, dim3((unsigned)ceil_div(cuts.rows, 16)), dim3(256),
                            0, s, p, g.gy, stats, cuts.rows);
      }))
    return e;
  auto sum = [&](auto keys, const Cut &c, const fdc_heads &out0, const fdc_heads &out1, int n, long long total) {
    return by_dtype(a.dtype, [&](auto tag) {
      return timed_launch("attn_sum", k_attn_sum<decltype(tag), decltype(keys)::value>,
                          dim3((unsigned)ceil_div(total, 256)), dim3(256), 0, s, p, (const float *)part, out0, out1, c.splits,
                          n, total);
    });
  };
  const Cut &q = cuts.q, &kv = cuts.kv;
  if (hipError_t e = by_shape(a.dtype, a.D, q.waves, [&](auto tag, auto dp, auto waves) {
        using T = decltype(tag);
        constexpr int DP = decltype(dp)::value, W = decltype(waves)::value;
        return launch_tiles<k_attn_bwd_q<T, DP, W>>("attn_bwd_q", (long long)a.B * a.G * q.tiles * q.splits, 64 * W,
                                                    4 * tile_bytes<T, DP>(), s, p, g.gy, g.gq, (const float2 *)stats, part,
                                                    q.tiles, q.splits, q.run);
      }))
    return e;
  if (q.splits > 1)
    if (hipError_t e = sum(std::false_type{}, q, g.gq, g.gq, p.R, cuts.rows * (p.D4 / 4))) return e;
  if (hipError_t e = by_shape(a.dtype, a.D, kv.waves, [&](auto tag, auto dp, auto waves) {
        using T = decltype(tag);
        constexpr int DP = decltype(dp)::value, W = decltype(waves)::value;
        return launch_tiles<k_attn_bwd_kv<T, DP, W>>(
            "attn_bwd_kv", (long long)a.B * a.G * kv.tiles * kv.splits, 64 * W,
            4 * tile_bytes<T, DP>() + 2 * attn_keys(sizeof(T)) * sizeof(float2), s, p, g.gy, g.gk, g.gv, (const float2 *)stats,
            part, kv.tiles, kv.splits, kv.run);
      }))
    return e;
  if (kv.splits > 1) return sum(std::true_type{}, kv, g.gk, g.gv, a.Lk, cuts.keys * (2 * p.D4 / 4));
  return hipSuccess;
}

}  // namespace fdc
