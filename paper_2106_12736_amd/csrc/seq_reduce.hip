// Sums of per-workgroup partial results of the sequence operators, in a fixed order.
#include "sequence.h"

namespace fdc {

// A workgroup sums 64 columns: wave g takes the rows g, g + W, ... in order (four loads in
// flight), then wave 0 adds the W sums in wave order.  A pass over `part` (HBM- or L2-bound).
template <int W>
__global__ __launch_bounds__(64 * W) void k_col_sums(const float *__restrict__ part, long long rows, long long cols,
                                                     ColSegments segs) {
  __shared__ float red[W][64];
  const int lane = threadIdx.x & 63, g = threadIdx.x >> 6;
  const long long c = (long long)blockIdx.x * 64 + lane;
  float s = 0.f;
  if (c < cols) {
    long long r = g;
    for (; r + 3 * W < rows; r += 4 * W) {
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = part[(r + i * W) * cols + c];
#pragma unroll
      for (int i = 0; i < 4; ++i) s += v[i];
    }
    for (; r < rows; r += W) s += part[r * cols + c];
  }
  if constexpr (W > 1) {
    red[g][lane] = s;
    __syncthreads();
    if (g != 0) return;
    s = red[0][lane];
#pragma unroll
    for (int i = 1; i < W; ++i) s += red[i][lane];
  }
  if (c >= cols) return;
  long long at = c;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    if (i >= segs.count) return;
    const ColSegment &q = segs.seg[i];
    if (at < q.cols) {
      if (q.out != nullptr) q.out[(at % q.inner) * q.mult + at / q.inner] = s;
      return;
    }
    at -= q.cols;
  }
}

hipError_t launch_col_sums(const float *part, long long rows, long long cols, const ColSegments &segs, hipStream_t s) {
  const long long blocks = ceil_div(cols, 64);
  if (blocks >= (1LL << 22)) return hipErrorInvalidValue;
  // many rows: 16 waves share the rows of 64 columns; few: 4
  if (rows > 64)
    return timed_launch("seq_col_sums", k_col_sums<16>, dim3((unsigned)blocks), dim3(1024), 0, s, part, rows, cols,
                        segs);
  return timed_launch("seq_col_sums", k_col_sums<4>, dim3((unsigned)blocks), dim3(256), 0, s, part, rows, cols, segs);
}

}  // namespace fdc
