// What the kernels of cross attention share (cross_attention.hip: forward, cross_attention_few.hip: forward for few rows,
// cross_attention_bwd_q.hip, cross_attention_bwd_kv.hip: backward).
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
#pragma once

#include <algorithm>

#include "device.h"
#include "lds_limit.h"
#include "sequence.h"

namespace fdc {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef short v4s __attribute__((ext_vector_type(4)));

namespace attention {

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
// A tile's rows are longer than their channels.  16-bit rows are an odd number of 4 words, so that 16-byte reads of a row a
// lane have no conflicts in LDS's banks (4 cycles; at 72 words instead of 76 they take 1.8 times as long).  The transposed
// reads take 4 cycles, of which half are counted as conflicts, and are what the kernels' conflicts come from (20 to 29 % of
// LDS's cycles); 16-byte writes of a tile take 8 (96 channels 10.6, 32 channels 15.9).  float32: the two reads of a row's 8
// values take 8 cycles each, half of them conflicts, columns 4 without.
template <class T, int DP>
constexpr int kStride = DP + (sizeof(T) == 4 ? 8 : DP == 32 || DP == 128 ? 24 : 8);
// LDS: two buffers of two tiles, and at its beginning and end 32 rows for each wave.
template <class T, int DP, int W>
constexpr size_t tiles_bytes() {
  return (size_t)(4 * attn_keys(sizeof(T)) > 32 * W ? 4 * attn_keys(sizeof(T)) : 32 * W) * kStride<T, DP> * sizeof(T);
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
// The rows row0 + l % 32 of a tile, `COUNT` steps of 16 channels from step `from` on.  A 16-bit product takes 32 cycles
// and its factor's way from LDS over 100, so that fragments are read some products ahead, and the order of reads and products
// is kept from being changed (ahead()); float32's eight instructions a product cover it.
template <class T, int DP, int COUNT>
struct Rows {
  Frag<T> f[COUNT];
  __device__ __forceinline__ void load(const T *tile, int row0, int from, int lane) {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) f[i] = row_frag<T, DP>(tile, row0 + (lane & 31), from + i, lane >> 5);
  }
};
// The columns of 32 rows of a tile from row0, all channels.
template <class T, int DP>
struct Columns {
  Frag<T> f[2][DP / 32];
  __device__ __forceinline__ void load(const T *tile, int row0, int lane) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) f[u][d] = column_frag<T, DP>(tile, row0 + 16 * u, 32 * d, lane);
  }
  // o[d] += the columns' products with 32 values of the other factor
  __device__ __forceinline__ void add_to(v16f (&o)[DP / 32], const Frag<T> (&e)[2]) const {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) mma(o[d], f[u][d], e[u]);
  }
};
template <class T>
__device__ __forceinline__ void ahead() {
  if constexpr (sizeof(T) == 2) __builtin_amdgcn_sched_barrier(0);
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

// A row's 16-byte piece that begins at channel c is read from first_of(c, D): its last one, where D is not a number of pieces,
// from V channels before the row's end, and is moved down to its place by move_pieces, 0 past the end.  So any width's loads
// are 16 bytes and all under way at once: read element by element the last pieces took up to half of a call's time (8 heads
// of 87 f16, 1178 rows on 11588 keys, 132 us, so 68).
template <class T>
__device__ __forceinline__ int first_of(int c, int D) {
  return min(c, D - 16 / (int)sizeof(T));
}
template <class T, int V>
__device__ __forceinline__ void move_piece(Pack<T, V> &x, int by) {
  constexpr int W = Pack<T, V>::W, E = V / W;
  const int words = by / E;
#pragma unroll
  for (int step = W / 2; step > 0; step /= 2)
#pragma unroll
    for (int i = 0; i < W; ++i) x.w[i] = words & step ? i + step < W ? x.w[i + step] : 0 : x.w[i];
  if constexpr (E == 2) {
#pragma unroll
    for (int i = 0; i < W; ++i) x.w[i] = by & 1 ? x.w[i] >> 16 | (i + 1 < W ? x.w[i + 1] << 16 : 0) : x.w[i];
  }
}
// A lane's pieces, under one branch (one for each slowed other widths by up to 9 %); rows of less than a piece are read in place.
template <class T, int V, int N, class Channel>
__device__ __forceinline__ void move_pieces(Pack<T, V> (&x)[N], int D, Channel &&channel) {
  if (D % V == 0 || D < V) return;
#pragma unroll
  for (int i = 0; i < N; ++i) move_piece(x[i], max(channel(i) + V - D, 0));
}
// A wave's 32 rows between memory and registers, through its own rows of LDS (`area`): memory is read and written in whole
// lines, 16 bytes a lane, a row's neighbours side by side.  Each lane knows where row l % 32 begins (`offset`, in elements
// from `base`) and whether it is there.
template <class T, int DP>
struct WaveRows {
  static constexpr int V = 16 / (int)sizeof(T), PR = DP / V, N = 32 * PR / 64, S = kStride<T, DP>;
  Pack<T, V> x[N];
  // wide: D is a 16-byte piece or more; rows that are not there are memory all the same.  What a kernel reads first is
  // issued before any of it is waited for.
  __device__ __forceinline__ void issue(const T *base, int64_t offset, int D, bool wide, bool there, int lane) {
    if (wide) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int row = (lane + 64 * i) / PR, c = (lane + 64 * i) % PR * V;
        x[i] = load_pack<T, V>(base + __shfl(offset, row, 64) + first_of<T>(c, D));
      }
    } else {
      const uint64_t live = __ballot(there);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int row = (lane + 64 * i) / PR, c = (lane + 64 * i) % PR * V;
        const int64_t at = __shfl(offset, row, 64);
        x[i] = Pack<T, V>{};
        if (c < D && (live >> row & 1)) x[i] = load_some<T, V>(base + at + c, D - c);
      }
    }
  }
  // f = the channels of row l % 32 as the factor of a product over channels, 0 where the row is not there.
  __device__ __forceinline__ void land(Frag<T> (&f)[DP / 16], T *area, int D, bool there, int lane) {
    const uint64_t live = __ballot(there);
    move_pieces(x, D, [&](int i) { return (lane + 64 * i) % PR * V; });
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = (lane + 64 * i) / PR, c = (lane + 64 * i) % PR * V;
      if (!(live >> row & 1) || c >= D) x[i] = Pack<T, V>{};
      *reinterpret_cast<Pack<T, V> *>(area + row * S + c) = x[i];
    }
    wave_sync();
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) f[i] = row_frag<T, DP>(area, lane & 31, i, lane >> 5);
    wave_sync();
  }
  // Row l % 32 = value(d, j), the lane's four channels 32 d + 8 j + 4 (l / 32) ..., rounded; `there`: whether it is written.
  template <class F>
  static __device__ __forceinline__ void store(T *area, T *base, int64_t offset, int D, bool there, int lane, F &&value) {
    const uint64_t live = __ballot(there);
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float4 x = value(d, j);
        const float y[4] = {x.x, x.y, x.z, x.w};
        store_pack<T, 4>(area + (lane & 31) * S + 32 * d + 8 * j + 4 * (lane >> 5), y);
      }
    wave_sync();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = (lane + 64 * i) / PR, c = (lane + 64 * i) % PR * V;
      const int64_t at = __shfl(offset, row, 64);
      const Pack<T, V> x = *reinterpret_cast<const Pack<T, V> *>(area + row * S + c);
      if (c >= D || !(live >> row & 1)) continue;
      if (c + V <= D) {
        __builtin_memcpy(base + at + c, &x, sizeof x);
      } else {
        const T *e = area + row * S + c;
#pragma unroll
        for (int k = 0; k < V; ++k)
          if (c + k < D) base[at + c + k] = e[k];
      }
    }
    wave_sync();
  }
};
template <int DP>
__device__ __forceinline__ float4 four(const v16f (&o)[DP / 32], int d, int j, float f) {
  return {o[d][4 * j] * f, o[d][4 * j + 1] * f, o[d][4 * j + 2] * f, o[d][4 * j + 3] * f};
}

// A tile on its way from memory to LDS, in 16-byte pieces of its rows; rows whose bit of `there` is not set are 0.
// Move: widths that are not a number of pieces are read as such, too.
template <class T, int DP, int TH, bool Move = true, int ROWS = attn_keys(sizeof(T))>
struct Staged {
  static constexpr int V = 16 / (int)sizeof(T), PR = DP / V, COUNT = ROWS * PR, N = (COUNT + TH - 1) / TH;
  Pack<T, V> x[N];
  static __device__ __forceinline__ int row_of(int i) { return ((int)threadIdx.x + i * TH) / PR; }
  static __device__ __forceinline__ int channel_of(int i) { return ((int)threadIdx.x + i * TH) % PR * V; }
  // at(i): where the row of piece i begins (memory whether the row is there or not)
  template <class At>
  __device__ __forceinline__ void load_whole(At &&at, int D) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = load_pack<T, V>(at(i) + first_of<T>(channel_of(i), D));
  }
  template <class At>
  __device__ __forceinline__ void load_parts(At &&at, int D, uint64_t there) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = channel_of(i);
      x[i] = Pack<T, V>{};
      if ((COUNT % TH == 0 || row_of(i) < COUNT / PR) && c < D && (there >> row_of(i) & 1))
        x[i] = load_some<T, V>(at(i) + c, D - c);
    }
  }
  static __device__ __forceinline__ bool in_whole(int D, bool wide) { return Move ? wide : D % V == 0; }
  template <class At>
  __device__ __forceinline__ void load(At &&at, int D, bool wide, uint64_t there) {
    if (in_whole(D, wide))
      load_whole(at, D);
    else
      load_parts(at, D, there);
  }
  __device__ __forceinline__ void store(T *tile, int D, uint64_t there) {
    if constexpr (Move) move_pieces(x, D, [&](int i) { return channel_of(i); });
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (!(there >> (row_of(i) & 63) & 1) || channel_of(i) >= D) x[i] = Pack<T, V>{};
      if (COUNT % TH == 0 || row_of(i) < COUNT / PR)
        *reinterpret_cast<Pack<T, V> *>(tile + row_of(i) * kStride<T, DP> + channel_of(i)) = x[i];
    }
  }
};

// What the kernels share of a call.
struct Attn {
  fdc_cross_attention_args a;
  int per, R;  // query heads a key head, rows a key head
  int D4;      // channels of a partial result's row
  float c;     // scale log2(e)
  bool wide;   // D is a 16-byte piece or more
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
  const int in = min(r, p.R - 1), hh = in / p.a.Lq, t = in - hh * p.a.Lq;
  return {g * p.per + hh, t, r < p.R && t < queries};
}
__device__ __forceinline__ int64_t offset_of(const fdc_heads &x, int b, int64_t t, int64_t h) {
  return b * x.batch_stride + t * x.token_stride + h * x.head_stride;
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

// ---- backward ----------------------------------------------------------------
// float16's probabilities are held 2^7 times as large, so that small ones keep their digits (2^-14 is its least normal
// number); they stay below 2^15 with the largest score up to 2^8 past the one they are taken relative to.
template <class T>
constexpr float kUp = std::is_same_v<T, _Float16> ? 7.f : 0.f;
constexpr float kLate = 8.f;

// What x's rounding loses, as it is kept.
template <class T>
__device__ __forceinline__ float low_of(float x) {
  return (x - (float)(T)x) * kLowUp<T>;
}

// Four channels c ... of a finished row r: its y, what that loses, and its lse, from the sums relative to m.
template <class T>
__device__ __forceinline__ void store_row_part(const Attn &p, int g, int b, int64_t at_row, int r, int queries, int c,
                                               float (&o)[4], float m, float l, float w) {
  const Row row = row_of(p, g, r, queries);
  const bool none = !row.live || l == 0.f;
  const float f = 1.f / w;
#pragma unroll
  for (int j = 0; j < 4; ++j) o[j] = none ? 0.f : o[j] * f;  // not by a product: o is NaN where a key it sees is
  store_some<T, 4>(at<T>(p.a.y, b, row.t, row.head) + c, o, p.a.D - c);
  if constexpr (sizeof(T) == 2) {
    if (p.low != nullptr) {
      const float rest[4] = {low_of<T>(o[0]), low_of<T>(o[1]), low_of<T>(o[2]), low_of<T>(o[3])};
      store_pack<T, 4>(static_cast<T *>(p.low) + at_row * p.D4 + c, rest);
    }
  }
  if (p.lse != nullptr && c == 0)
    p.lse[at_row] = none ? -INFINITY : (m + __builtin_amdgcn_logf(l) - kUp<T>) * kLn2;
}

// float16's probabilities times 2^15 (at most 2^15): 2^-14 is its least normal number.
template <class T>
constexpr float kUpBack = std::is_same_v<T, _Float16> ? 15.f : 0.f;

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

// ---- host ----------------------------------------------------------------------
// Workgroups of `waves` waves that have 32 rows (or keys) each, and runs of the tiles they go through.
struct Cut {
  int waves, tiles, splits, run;
};
// together: how many workgroups of four waves a compute unit holds.
inline Cut cut(long long heads, long long own, long long through, int tile, bool eight, int together) {
  Cut c;
  c.waves = eight && own > 192 ? 8 : own > 64 ? 4 : 2;
  c.tiles = (int)ceil_div(own, 32 * c.waves);
  // as many as run at once on 256 compute units, not more: what is left over would take as long as the first round
  const long long steps = ceil_div(through, tile), blocks = heads * c.tiles, most = 256 * (c.waves == 8 ? 1 : together);
  const long long splits = std::max(1LL, std::min(most / blocks, steps / 2));
  c.run = (int)ceil_div(steps, splits);
  c.splits = (int)ceil_div(steps, c.run);
  return c;
}
// Waves of a workgroup of the form for few rows: two a SIMD, and one with float32 heads of more than 32 channels, whose
// registers allow no more.
template <class T>
constexpr int few_waves(int DP) {
  return sizeof(T) == 2 ? 8 : DP <= 32 ? 8 : 4;
}
constexpr int kFewRows = 32;
// Runs of blocks of 32 keys: one launch where a workgroup's keys are at most 512 KB or there are two workgroups for every
// compute unit, else runs of at least two blocks a wave.  A call in one launch and in runs, in a captured graph, us: bf16 of
// 512 KB a head, 16 heads of 64 channels 15.6 and 11.5, 64 of 128 15.9 and 16.3, 256 of 128 27.9 and 35.7; of 1 MB 26.1 and
// 10.9, 23.8 and 22.9, 45.6 and 55.1.  float32 of 256 KB, 16 heads of 64 18.6 and 14.6; of 512 KB 31.8 and 15.7, 64 of 128
// 31.2 and 22.9, 256 of 128 34.9 and 45.9; of 1 MB 58.4 and 15.0, 54.9 and 27.5, 58.8 and 70.2.  So few heads of float32 would
// have runs from 256 KB on, and 256 heads none at all.
inline Cut cut_few(int dtype, long long heads, long long keys, int D) {
  Cut c;
  const int DP = D <= 32 ? 32 : D <= 64 ? 64 : D <= 96 ? 96 : 128;
  c.waves = dtype_size(dtype) == 2 ? few_waves<short>(DP) : few_waves<float>(DP);
  c.tiles = 1;
  const long long blocks = ceil_div(keys, 32), bytes = keys * D * 2 * (long long)dtype_size(dtype);
  long long splits = 1;
  if (bytes > (512 << 10)) splits = std::max(1LL, std::min(ceil_div(512, heads), blocks / (2 * c.waves)));
  c.run = (int)ceil_div(blocks, splits);
  c.splits = (int)ceil_div(blocks, c.run);
  return c;
}
struct Cuts {
  bool few;
  Cut fwd, q, kv;
  long long rows, keys, D4;
  Cuts(int dtype, int B, int Lq, int Lk, int H, int G, int D) {
    const long long heads = (long long)B * G, R = (long long)H / G * Lq;
    const int tile = attn_keys(dtype_size(dtype));
    // float32's factors are twice as many registers: eight waves of 256 hold 64 channels
    const bool eight = dtype_size(dtype) == 2 || D <= 64;
    q = cut(heads, R, Lk, tile, eight, eight ? 2 : 1);
    few = R <= kFewRows;
    fwd = few ? cut_few(dtype, heads, Lk, D) : q;
    kv = cut(heads, Lk, R, tile, D <= 64, D <= 64 ? 2 : 1);
    rows = heads * R, keys = heads * Lk, D4 = ceil_div(D, 4) * 4;
  }
  size_t fwd_floats() const { return fwd.splits > 1 ? (size_t)fwd.splits * rows * (D4 + 4) : 0; }
  size_t stats_floats() const { return (size_t)ceil_div(rows * 2, 4) * 4; }
  size_t q_floats() const { return q.splits > 1 ? (size_t)q.splits * rows * D4 : 0; }
  size_t kv_floats() const { return kv.splits > 1 ? (size_t)kv.splits * keys * 2 * D4 : 0; }
};

inline int64_t lse_floats(int B, int Lq, int H) { return ceil_div((int64_t)B * Lq * H, 4) * 4; }
inline Attn attn_of(const fdc_cross_attention_args &a, float *saved) {
  void *low = saved != nullptr && dtype_size(a.dtype) == 2 ? saved + lse_floats(a.B, a.Lq, a.H) : nullptr;
  return {a, a.H / a.G, a.H / a.G * a.Lq, (a.D + 3) / 4 * 4, a.scale * kLog2e, a.D * dtype_size(a.dtype) >= 16, saved, low};
}

// f(T{}, padded channels, waves) for the type, channels and waves of a call; `Eight`: eight waves with 16-bit heads of over 64
// channels, too.
template <bool Eight, class F>
hipError_t by_shape(int dtype, int D, int waves, F &&f) {
  using std::integral_constant;
  return by_dtype(dtype, [&](auto tag) {
    auto with = [&](auto dp) {
      if constexpr ((Eight && sizeof(tag) == 2) || decltype(dp)::value <= 64)
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

}  // namespace attention

// The forward for few rows, in cross_attention_few.hip, and the parts of the backward, in cross_attention_bwd_*.hip.
hipError_t launch_attention_few(const attention::Attn &p, const attention::Cut &c, float *part, hipStream_t s);
hipError_t launch_attention_bwd_q(const attention::Attn &p, const attention::Cut &c, const fdc_heads &gy, const fdc_heads &gq,
                                  float2 *stats, float *part, hipStream_t s);
hipError_t launch_attention_bwd_kv(const attention::Attn &p, const attention::Cut &c, const fdc_heads &gy,
                                   const fdc_heads &gk, const fdc_heads &gv, const float2 *stats, float *part,
                                   hipStream_t s);

}  // namespace fdc
