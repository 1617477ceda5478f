// Internal interface of the sequence operators (causal_conv.hip, scan.hip, block_norm.hip,
// distill.hip, seq_reduce.hip) and the device helpers they share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "fdc.h"
#include "internal.h"

namespace fdc {

// ---- host ------------------------------------------------------------------
inline size_t dtype_size(int dtype) { return dtype == FDC_F32 ? 4 : 2; }

constexpr int kConvMaxTaps = 8;
constexpr int kScanMaxStates = 64;
constexpr int kScanBlock = 16;  // tokens between two saved states
constexpr int kNormMaxWidth = 8192;
constexpr int kDistillMaxTeacher = 1024;
constexpr int kDistillStats = 5;  // floats a row that the forward keeps for the backward

hipError_t launch_causal_conv_fwd(const fdc_causal_conv_args &a, hipStream_t s);
size_t causal_conv_bwd_ws(int dtype, int B, int L, int D, int n);  // bytes
hipError_t launch_causal_conv_bwd(const fdc_causal_conv_args &a, const fdc_tokens &gy, const fdc_tokens &gx, float *gw,
                                  float *gbias, float *part, hipStream_t s);

size_t scan_saved_floats(int B, int L, int D, int N);
size_t scan_fwd_ws_floats(int B, int L, int D, int N, int G);
size_t scan_bwd_ws_floats(int B, int L, int D, int N, int G);
hipError_t launch_scan_fwd(const fdc_scan_args &a, float *saved, float *ws, hipStream_t s);
hipError_t launch_scan_bwd(const fdc_scan_args &a, const float *saved, const fdc_scan_grads &g, float *ws,
                           hipStream_t s);
hipError_t launch_scan_step(const fdc_scan_args &a, hipStream_t s);

hipError_t launch_block_norm_fwd(const fdc_block_norm_args &a, void *out, int64_t out_stride, void *n,
                                 int64_t n_stride, float *stats, hipStream_t s);
size_t block_norm_bwd_ws_floats(int64_t R, int D);
hipError_t launch_block_norm_bwd(const fdc_block_norm_args &a, const float *stats, const fdc_block_norm_grads &g,
                                 float *part, hipStream_t s);

size_t distill_ws_floats(int dtype, int64_t R, int V);
// gloss and gz NULL: the loss alone.
hipError_t launch_distill(const fdc_distill_args &a, float *loss, float *stats, const float *gloss, void *gz,
                          int64_t gz_stride, float *ws, hipStream_t s);
hipError_t launch_distill_bwd(const fdc_distill_args &a, const float *stats, const float *gloss, void *gz,
                              int64_t gz_stride, hipStream_t s);

// Sums over the rows of part [rows][cols] in row order, in segments of columns: column c of
// segment i goes to out[i][(c % inner[i]) * mult[i] + c / inner[i]] (out NULL: dropped).
struct ColSegment {
  float *out;
  int cols, inner, mult;
};
struct ColSegments {
  ColSegment seg[3];
  int count;
};
hipError_t launch_col_sums(const float *part, long long rows, long long cols, const ColSegments &segs, hipStream_t s);

// f(T{}) with the C++ type of a dtype.
template <class F>
auto by_dtype(int dtype, F &&f) {
  if (dtype == FDC_F32) return f(float{});
  if (dtype == FDC_BF16) return f(__bf16{});
  return f(_Float16{});
}

inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// ---- device ----------------------------------------------------------------
#ifdef __HIPCC__

// V consecutive elements in 32-bit words as they lie in memory (16-bit elements stay two a register).
template <class T, int V>
struct Pack {
  static constexpr int W = V * (int)sizeof(T) / 4;
  unsigned w[W];
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 4) {
      return __uint_as_float(w[i]);
    } else if constexpr (std::is_same_v<T, __bf16>) {
      return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    } else {
      const unsigned short h = (unsigned short)(i % 2 ? w[i / 2] >> 16 : w[i / 2]);
      return (float)__builtin_bit_cast(_Float16, h);
    }
  }
};
template <class T>
__device__ __forceinline__ unsigned element_bits(T v) {
  if constexpr (sizeof(T) == 4)
    return __float_as_uint(v);
  else
    return __builtin_bit_cast(unsigned short, v);
}
// From and to any element-aligned address (16-byte global accesses need no alignment beyond the
// element's on this hardware).
template <class T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(const T *p) {
  Pack<T, V> x;
  __builtin_memcpy(&x, p, sizeof x);
  return x;
}
template <class T, int V>
__device__ __forceinline__ void store_pack(T *p, const float (&f)[V]) {
  struct {
    T v[V];
  } x;
#pragma unroll
  for (int i = 0; i < V; ++i) x.v[i] = (T)f[i];
  __builtin_memcpy(p, &x, sizeof x);
}
// The first n (>= 1) of V elements; the others are `fill`.
template <class T, int V>
__device__ __forceinline__ Pack<T, V> load_some(const T *p, int n, float fill = 0.f) {
  if (n >= V) return load_pack<T, V>(p);
  constexpr int E = 4 / sizeof(T);  // elements a word
  Pack<T, V> x;
#pragma unroll
  for (int j = 0; j < Pack<T, V>::W; ++j) {
    x.w[j] = 0;
#pragma unroll
    for (int i = 0; i < E; ++i)
      x.w[j] |= element_bits<T>(j * E + i < n ? p[j * E + i] : (T)fill) << (i * 8 * (int)sizeof(T) % 32);
  }
  return x;
}
template <class T, int V>
__device__ __forceinline__ void store_some(T *p, const float (&f)[V], int n) {
  if (n >= V) {
    store_pack<T, V>(p, f);
    return;
  }
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i < n) p[i] = (T)f[i];
}

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
__device__ __forceinline__ float rcp_fast(float x) { return __builtin_amdgcn_rcpf(x); }
// 1 / (1 + exp(-x)): exp overflows to infinity for very negative x, and the quotient is 0.
__device__ __forceinline__ float sigmoid(float x) { return rcp_fast(1.f + exp_fast(-x)); }
// log(1 + exp(x)): x + log(1 + exp(-x)) for positive x.  With e = exp(-|x|) and w = 1 + e rounded, e - (w - 1)
// is what the rounding of w lost, and log(1 + e) = log(w) + that / w; where it matters w is 1 (the
// neglected part is at most 2^-24 e), so that small results keep their relative precision.
__device__ __forceinline__ float softplus(float x) {
  const float e = exp_fast(-fabsf(x)), w = 1.f + e;
  return fmaxf(x, 0.f) + fmaf(kLn2, __builtin_amdgcn_logf(w), e - (w - 1.f));
}
// The length of sequence b, within [0, L].
__device__ __forceinline__ int length_of(const int *lengths, int b, int L) {
  if (lengths == nullptr) return L;
  const int n = lengths[b];
  return n < 0 ? 0 : n > L ? L : n;
}

// Data in LDS that one lane of a wave writes and another lane of the same wave reads.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <int Ctrl>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), Ctrl, 0xf, 0xf, true));
}
// Sum over groups of LN adjacent lanes (LN <= 16: within a row of 16 lanes); every lane gets it.
template <int LN>
__device__ __forceinline__ float lane_sum(float v) {
  if constexpr (LN >= 2) v += dpp<0xB1>(v);   // lane ^ 1
  if constexpr (LN >= 4) v += dpp<0x4E>(v);   // lane ^ 2
  if constexpr (LN >= 8) v += dpp<0x141>(v);  // mirrored in 8: the other four
  if constexpr (LN >= 16) v += dpp<0x140>(v);  // mirrored in 16: the other eight
  return v;
}
// The value of lane S of each group of LN adjacent lanes.
template <int LN, int S>
__device__ __forceinline__ float lane_bcast(float v) {
  static_assert(S < LN);
  if constexpr (LN == 1) return v;
  if constexpr (LN == 2) return dpp<(S | S << 2 | (2 + S) << 4 | (2 + S) << 6)>(v);
  if constexpr (LN == 4) return dpp<S * 0x55>(v);
  // and-mask 0x1f & ~(LN - 1), or-mask S within 32 lanes
  if constexpr (LN == 8) return __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(v), 0x18 | S << 5));
  if constexpr (LN == 16) return __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(v), 0x10 | S << 5));
  return 0.f;
}
// Sum and maximum over the 64 lanes; every lane gets it (same order in every lane).
__device__ __forceinline__ float wave_sum(float v) {
  v = lane_sum<16>(v);
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
  return v;
}

template <class F, int... I>
__device__ __forceinline__ void static_for_impl(F &&f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
// f(integral_constant<0>) ... f(integral_constant<Count - 1>)
template <int Count, class F>
__device__ __forceinline__ void static_for(F &&f) {
  static_for_impl(static_cast<F &&>(f), std::make_integer_sequence<int, Count>{});
}

#endif  // __HIPCC__

}  // namespace fdc
