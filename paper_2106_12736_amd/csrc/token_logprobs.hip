// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and their gradient.
//
//   with d = (z - m) / tau, m the row's largest logit, s = sum exp(d), u = sum exp(d) d:
//   l[v] = d[v] - log s,   entropy = log s - u / s  (two terms that are not negative: nothing cancels)
//   gz[v] = 1/tau ([v = token] glogp + sum_k [v = idx_k] gtop_k - p[v] (glogp + sum gtop) - gentropy p[v] (l[v] + entropy))
//
// The forward is one pass over z: a workgroup goes through a row, or a segment of one, in chunks of four 16-byte pieces a
// thread, the next chunk's loads under way; every thread holds the running maximum and sums of its own logits, which
// are joined at the end.  The K best: of the first chunk every thread's largest logit is known, and the K-th
// largest of these is a lower bound of the K-th best (K threads have one that large), below which all but a few more
// than K logits lie; those above go to LDS, where each finds its place by counting the ones before it.  From then on only
// logits above the K-th best so far are looked at (a chunk's largest logit tells whether there are any), K / j of the
// j-th chunk where they come in no order.  Where too many lie above (many equal logits, rising ones), the bound is raised by
// bisection until few enough do; equal logits are told apart by their places.
//
// Many rows: a workgroup each; few rows: segments, joined by a workgroup a row.
//
// 4096 x 32000 bf16 without alternatives 52 us (5.0 TB/s; 71 behind a gradient's writes), 2048 x 100000 with 64 of them 129
// us (3.2 TB/s), of which the first chunk's bound and the last ranking are some 20 us and later candidates 25: there the
// vector units are busy 85 % of the time (7 registers spilled).  With the rows in registers whole, and every segment's K best found anew, it
// took 393 us.  Candidates taken from registers instead of read again took 134.  The gradient, 4096 x 32000 bf16, 117 us
// (4.5 TB/s).
#include <algorithm>

#include "sequence.h"

namespace fdc {

namespace {

constexpr int kMost = 512;  // candidates in LDS
constexpr float kLowest = -3.402823466e38f;

template <class T>
constexpr int kLogitV = 16 / (int)sizeof(T);

// Keys of the same order as the logits, -0 as 0, NaN above all.
__device__ __forceinline__ uint32_t key_of(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t b = __float_as_uint(x + 0.f);
  return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu)); }
constexpr uint32_t kInfKey = 0xff800000u;
// A logit and its place: larger logits first, then lower places.  0 stands for none.
__device__ __forceinline__ uint64_t pair_of(uint32_t key, int place) { return (uint64_t)key << 32 | ~(uint32_t)place; }
__device__ __forceinline__ int place_of(uint64_t pair) { return (int)~(uint32_t)pair; }

// With t = (z - m) c, c = log2(e) / tau: s = sum 2^t, u = sum 2^t t.
struct Sums {
  float m, s, u;
  // s and u relative to t + by
  __device__ __forceinline__ void shift(float by) {
    const float f = exp2_fast(by);
    s *= f;
    u = fmaf(s, by, u * f);  // the sum scaled first: segments of the type's lowest value
  }
};
// (from - to) c as a number.
__device__ __forceinline__ float distance(float from, float to, float c) {
  return from == to ? 0.f : fmaxf((from - to) * c, kLowest);
}
__device__ __forceinline__ void add(Sums &a, Sums b, float c) {
  if (b.s == 0.f) return;  // nothing but -inf
  if (a.s == 0.f) {
    a = b;
    return;
  }
  const float m = fmaxf(a.m, b.m);
  a.shift(distance(a.m, m, c));
  b.shift(distance(b.m, m, c));
  a = {m, a.s + b.s, a.u + b.u};
}

// The largest logits that a first bound is found from: of every thread, or of four adjacent ones.
template <int TH>
constexpr int kMaxima = TH < 256 ? TH : 256;

template <int TH>
struct TopScratch {
  uint32_t maxima[kMaxima<TH>];
  uint64_t found[2][kMost];
  int count;
  uint32_t bound;
  int red[2][TH / 64];
};

// By one wave: a key that at least K of the maxima are not below, few of them if there is one (0: all).
template <int TH>
__device__ __forceinline__ uint32_t bound_of(const uint32_t *maxima, int K, int lane) {
  constexpr int N = kMaxima<TH> / 64;
  if (K > kMaxima<TH>) return 0;
  uint32_t mine[N], bound = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) mine[i] = maxima[i * 64 + lane];
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t tried = bound | 1u << bit;
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) n += __popcll(__ballot(mine[i] >= tried));
    if (n < K) continue;
    bound = tried;
    if (n <= K + K / 8) break;
  }
  return bound;
}

// The sum of n over the workgroup; `turn` counts the calls (two sets of partial sums in turn: one barrier each).
template <int TH>
__device__ __forceinline__ int count_all(TopScratch<TH> &t, int n, int turn) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) n += __shfl_xor(n, off, 64);
  if ((threadIdx.x & 63) == 0) t.red[turn & 1][threadIdx.x >> 6] = n;
  __syncthreads();
  int sum = 0;
#pragma unroll
  for (int i = 0; i < TH / 64; ++i) sum += t.red[turn & 1][i];
  return sum;
}

// The logits that are not below a bound: above f, or equal to it and at places up to `last`; NaN is above all, and with `odd`
// itself the bound.
struct Bound {
  float f;
  bool odd;
  int last;
  __device__ __forceinline__ Bound(uint32_t key, int last_) : last(last_) {
    odd = key > kInfKey;
    f = key < ~kInfKey ? -INFINITY : of_key(key);
  }
  __device__ __forceinline__ bool has(float x, int place) const {
    const bool early = place <= last, nan = x != x;
    return (nan & (early | !odd)) | (!odd & ((x > f) | ((x == f) & early)));
  }
};

// Adds a chunk's logits from the bound on to t.found[set], which holds `kept`, at least the K best of them where they are
// too many, and returns how many it holds.  `bound` and t.count (kept) have been written before a barrier.  The chunk is
// z[from] ... z[end - 1]; largest: the thread's largest, odd: it has NaN; above(f, put) calls put(logit, place) for the thread's
// logits that are not below f.  What is rare reads the chunk again, so that the registers are those of the common way.
template <class T, int TH, class Above>
__device__ __forceinline__ int add_top(TopScratch<TH> &t, int set, int kept, uint32_t bound, int K, float largest, bool odd,
                                       const T *z, int from, int end, Above &&above) {
  auto put = [&](float x, int place) {
    const int at = atomicAdd(&t.count, 1);
    if (at < kMost) t.found[set][at] = pair_of(key_of(x), place);
  };
  auto each = [&](auto &&f) {
    for (int at = from + (int)threadIdx.x; at < end; at += TH) f((float)z[at], at);
  };
  const Bound first(bound, end - 1);
  if (first.odd || first.f == -INFINITY)
    each([&](float x, int place) {
      if (first.has(x, place)) put(x, place);
    });
  else if (odd || largest >= first.f)
    above(first.f, put);
  __syncthreads();
  int n = t.count;
  if (n <= kMost) return n;
  // bisection: K or more logits of the chunk are not below lo, fewer than K not below hi
  const int most = kMost - kept;
  n -= kept;
  uint32_t most_key = odd ? 0xffffffffu : key_of(largest);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) most_key = max(most_key, (uint32_t)__shfl_xor((int)most_key, off, 64));
  if ((threadIdx.x & 63) == 0) t.red[1][threadIdx.x >> 6] = (int)most_key;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < TH / 64; ++i) most_key = max(most_key, (uint32_t)t.red[1][i]);
  uint64_t lo = bound, hi = (uint64_t)most_key + 1;
  int turn = 0;
  auto count = [&](const Bound &b) {
    int c = 0;
    each([&](float x, int place) { c += b.has(x, place); });
    return count_all(t, c, turn++);
  };
  while (hi - lo > 1 && n > most) {
    const uint32_t mid = (uint32_t)((lo + hi) / 2);
    const int c = count(Bound(mid, end - 1));
    if (c >= K)
      lo = mid, n = c;
    else
      hi = mid;
  }
  // too many equal ones: the places up to `last` are enough
  int none = 0, last = end - 1;  // the places below `none` are too few
  while (last > none && n > most) {
    const int mid = none + (last - none) / 2, c = count(Bound((uint32_t)lo, mid));
    if (c >= K)
      last = mid, n = c;
    else
      none = mid + 1;
  }
  __syncthreads();
  if (threadIdx.x == 0) t.count = kept;
  __syncthreads();
  const Bound b((uint32_t)lo, last);
  each([&](float x, int place) {
    if (b.has(x, place)) put(x, place);
  });
  __syncthreads();
  return min(t.count, kMost);
}

// put(rank, pair) for the K best of n pairs, each from one thread.
template <int TH, class Put>
__device__ __forceinline__ void rank_top(const uint64_t *found, int n, int K, Put &&put) {
  for (int i = threadIdx.x; i < n; i += TH) {
    const uint64_t mine = found[i];
    int rank = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) rank += found[j] > mine;
    if (rank < K) put(rank, mine);
  }
}

struct Result {
  float m, s, log_s, per;  // per: 1 / tau
  __device__ __forceinline__ Result(const Sums &x, float tau) {
    m = x.m, s = x.s, log_s = __builtin_amdgcn_logf(x.s) * kLn2, per = 1.f / tau;
  }
  __device__ __forceinline__ float logp(float z) const { return (z - m) * per - log_s; }
};

// By one thread: what a row's sums say, but for its alternatives.
template <class T>
__device__ __forceinline__ void row_result(const fdc_token_logprobs_args &a, int64_t row, const Sums &x, float *logp,
                                           float *entropy, float *stats) {
  const Result r(x, a.tau);
  const float h = r.log_s - x.u / x.s * kLn2;
  if (logp != nullptr) {
    const int v = a.tokens[row];
    logp[row] = v < 0 ? 0.f : v >= a.V ? NAN : r.logp((float)static_cast<const T *>(a.z)[row * a.z_stride + v]);
  }
  if (entropy != nullptr) entropy[row] = h;
  if (stats != nullptr) {
    float *p = stats + kLogprobStats * row;
    p[0] = x.m, p[1] = x.s, p[2] = h;
  }
}

// What a call writes.
struct Out {
  float *logp, *entropy;
  int32_t *idx;
  float *top, *stats;
  float4 *part;     // [R][segments]: m, s, u of a segment
  uint64_t *pairs;  // [R][segments][K]
};

// Keeps the compiler from holding what one pass over the pieces forms of them (floats, keys) for the next.
template <class T, int V>
__device__ __forceinline__ void keep_packed(Pack<T, V> &x) {
  asm volatile("" : "+v"(x.w[0]), "+v"(x.w[1]), "+v"(x.w[2]), "+v"(x.w[3]));
}

// Rows of many chunks want as many waves as there are; float16 with alternatives has 57 registers spilled at eight.
template <class T, int TH, int NV, bool Top>
constexpr int kWavesASimd = NV == 1 ? 1 : TH == 256 && Top && std::is_same_v<T, _Float16> ? 6 : 8;

// A workgroup a segment (of `seg` logits, `segs` a row).
template <class T, int TH, int NV, bool Top>
__global__ __launch_bounds__(TH, (kWavesASimd<T, TH, NV, Top>)) void k_logprobs(fdc_token_logprobs_args a, Out out, int seg, int segs) {
  constexpr int V = kLogitV<T>, W = TH / 64, CHUNK = TH * NV * V;
  __shared__ float rmax[W], rs[W], ru[W];
  __shared__ std::conditional_t<Top, TopScratch<TH>, int> scratch;
  const int64_t id = (int64_t)blockIdx.y * 32768 + blockIdx.x;
  const int64_t row = id / segs;
  if (row >= a.R) return;
  const int begin = (int)(id - row * segs) * seg, end = min(a.V, begin + seg);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float c = kLog2e / a.tau;
  const T *z = static_cast<const T *>(a.z) + row * a.z_stride;
  // A piece past the end is all -inf; one that the end lies in begins earlier, V logits before the end, and what belongs to
  // another piece of it is -inf.  (Rows of less than a piece have one, loaded logit by logit.)
  auto place_of_piece = [&](int at) { return TH == 64 || at + V <= end ? at : end - V; };
  auto load = [&](Pack<T, V>(&x)[NV], int from) {
    const unsigned none = sizeof(T) == 4 ? element_bits<T>((T)-INFINITY) : element_bits<T>((T)-INFINITY) * 0x10001u;
    if (from + CHUNK <= end) {
#pragma unroll
      for (int k = 0; k < NV; ++k) x[k] = load_pack<T, V>(z + from + (k * TH + tid) * V);
    } else if constexpr (TH == 64) {
      const int n = end - from - tid * V;
      x[0] = {none, none, none, none};
      if (n > 0) x[0] = load_some<T, V>(z + from + tid * V, n, -INFINITY);
    } else {
#pragma unroll
      for (int k = 0; k < NV; ++k) x[k] = load_pack<T, V>(z + place_of_piece(from + (k * TH + tid) * V));
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int at = from + (k * TH + tid) * V, skip = min(V, at - place_of_piece(at));
        constexpr int E = 4 / (int)sizeof(T);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (i * E < skip) x[k].w[i] = E == 2 && i * E + 1 >= skip ? (x[k].w[i] & 0xffff0000u) | (none & 0xffffu) : none;
        }
      }
    }
  };
  Pack<T, V> x[NV], next[NV];
  load(x, begin);
  Sums t{-INFINITY, 0.f, 0.f};
  // As long as a wave's logits are numbers and its maxima's m c at most 2^20, t is fma(z, c, -mc), with mc the rounded m c: off
  // by its rounding of at most 2^-5, which all of the thread's terms have in common and which is made good at the end.  Else
  // (z - m) c, held above -inf.  The second form for all: 4096 x 32000 without alternatives 50.5 us in place of 48.6 (bf16),
  // 49.9 in place of 47.0 (f16); 2048 x 100000 with 64 of them 121 in place of 125 (bf16), 138 in place of 132 (f16).
  float mc = -INFINITY;
  const float near = fminf(0x1p20f / c, -kLowest);
  bool careful = false;  // the same in every lane
  auto to_exact = [&] {
    if (t.s != 0.f) t.shift(fmaf(-t.m, c, mc));
  };
  int kept = 0, set = 0;
  uint32_t bound = 0;
  for (int from = begin; from < end; from += CHUNK) {
    const bool more = from + CHUNK < end;
    if (more) load(next, from + CHUNK);
    float best[NV], largest = -INFINITY;  // of each piece, and of all
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      best[k] = x[k].at(0);
#pragma unroll
      for (int i = 1; i < V; ++i) best[k] = fmaxf(best[k], x[k].at(i));
      largest = fmaxf(largest, best[k]);
    }
    if constexpr (Top) {
      if (from == begin) {
        if constexpr (TH == 1024) {
          float four = fmaxf(largest, dpp<0xB1>(largest));
          four = fmaxf(four, dpp<0x4E>(four));
          if (tid % 4 == 0) scratch.maxima[tid / 4] = key_of(four);
        } else {
          scratch.maxima[tid] = key_of(largest);
        }
        if (tid == 0) scratch.count = 0;
        __syncthreads();
        if (wave == W - 1) {
          const uint32_t b = bound_of<TH>(scratch.maxima, a.K, lane);
          if (lane == 0) scratch.bound = b;
        }
      }
    }
    if (!careful && __any(fabsf(largest) > near)) {
      to_exact();
      careful = true;
    }
    if (largest > t.m) {
      const float to = largest * c;
      if (t.s != 0.f) t.shift(careful ? distance(t.m, largest, c) : mc - to);
      t.m = largest, mc = to;
    }
    if (!careful) {
      const Sums before = t;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        keep_packed(x[k]);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float d = fmaf(x[k].at(i), c, -mc), e = exp2_fast(d);
          t.s += e;
          t.u = fmaf(e, d, t.u);
        }
        asm volatile("" : "+v"(t.s), "+v"(t.u));  // a piece at a time: its floats die with it
      }
      if (__any(t.u != t.u && t.s == t.s)) {  // 0 times -inf
        t = before;
        to_exact();
        careful = true;
      }
    }
    if (careful) {
      // of -inf alone so far (or with NaN): each term is 0 (or NaN)
      const float base = t.m == -INFINITY ? 0.f : t.m;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        keep_packed(x[k]);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float d = (x[k].at(i) - base) * c, e = exp2_fast(d);
          t.s += e;
          t.u = fmaf(e, fmaxf(d, kLowest), t.u);
        }
        asm volatile("" : "+v"(t.s), "+v"(t.u));
      }
    }
    if constexpr (Top) {
      if (from == begin) {
        __syncthreads();
        bound = scratch.bound;
      }
      const bool odd = t.s != t.s;
      if (__syncthreads_or(odd || largest >= Bound(bound, 0).f)) {
        // the few pieces that have one are read again (their registers cannot be chosen by number)
        auto above = [&](float f, auto &&put) {
          uint32_t pieces = 0;
#pragma unroll
          for (int k = 0; k < NV; ++k) pieces |= odd || best[k] >= f ? 1u << k : 0u;
          while (pieces != 0) {
            const int at = from + (__builtin_ctz(pieces) * TH + tid) * V, base = place_of_piece(at);
            pieces &= pieces - 1;
            const Pack<T, V> y = TH == 64 ? load_some<T, V>(z + base, end - base, -INFINITY) : load_pack<T, V>(z + base);
#pragma unroll
            for (int i = 0; i < V; ++i)
              if (!(y.at(i) < f) && base + i >= at && base + i < end) put(y.at(i), base + i);
          }
        };
        const int n = add_top<T, TH>(scratch, set, kept, bound, a.K, largest, odd, z, from, min(end, from + CHUNK), above);
        kept = n;
        // the K best so far, and the K-th as the bound: later logits have to be above it
        if (n > a.K + 64 || (from == begin && n >= a.K && more)) {
          rank_top<TH>(scratch.found[set], n, a.K, [&](int rank, uint64_t pair) {
            scratch.found[set ^ 1][rank] = pair;
            if (rank == a.K - 1) {
              const uint32_t key = (uint32_t)(pair >> 32);
              scratch.bound = key == 0xffffffffu ? key : key + 1;
            }
          });
          kept = a.K;
          set ^= 1;
          __syncthreads();
          bound = scratch.bound;
          if (tid == 0) scratch.count = kept;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) x[k] = next[k];
  }
  // the threads' sums, relative to the largest of all
  if (!careful) to_exact();
  float m = wave_max(t.m);
  if (lane == 0) rmax[wave] = m;
  __syncthreads();
  m = rmax[0];
#pragma unroll
  for (int w = 1; w < W; ++w) m = fmaxf(m, rmax[w]);
  if (t.m != m && !(t.s == 0.f)) t.shift(t.m == -INFINITY ? 0.f : distance(t.m, m, c));
  t.m = m;
  t.s = wave_sum(t.s);
  t.u = wave_sum(t.u);
  if (lane == 0) rs[wave] = t.s, ru[wave] = t.u;
  __syncthreads();
  t.s = t.u = 0.f;
#pragma unroll
  for (int w = 0; w < W; ++w) t.s += rs[w], t.u += ru[w];
  if (tid == 0) {
    if (segs == 1)
      row_result<T>(a, row, t, out.logp, out.entropy, out.stats);
    else
      out.part[id] = {t.m, t.s, t.u, 0.f};
  }
  if constexpr (Top) {
    const uint64_t *found = scratch.found[set];
    if (segs == 1) {
      const Result r(t, a.tau);
      rank_top<TH>(found, kept, a.K, [&](int rank, uint64_t pair) {
        out.idx[row * a.K + rank] = place_of(pair);
        out.top[row * a.K + rank] = r.logp(of_key((uint32_t)(pair >> 32)));
      });
    } else {
      uint64_t *to = out.pairs + id * a.K;
      rank_top<TH>(found, kept, a.K, [&](int rank, uint64_t pair) { to[rank] = pair; });
      for (int k = kept + tid; k < a.K; k += TH) to[k] = 0;  // a segment of less than K
    }
  }
}

// A workgroup a row: its segments' sums in order, and the best of their K best.
template <class T>
__global__ __launch_bounds__(256) void k_logprobs_join(fdc_token_logprobs_args a, Out out, int segs) {
  __shared__ TopScratch<256> t;
  __shared__ Sums all;
  const int64_t row = (int64_t)blockIdx.y * 32768 + blockIdx.x;
  if (row >= a.R) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const float c = kLog2e / a.tau;
  const uint64_t *pairs = out.pairs + row * segs * a.K;
  const int total = segs * a.K;
  uint64_t mine = 0;
  for (int i = tid; i < total; i += 256) mine = max(mine, pairs[i]);
  t.maxima[tid] = (uint32_t)(mine >> 32);
  if (tid == 0) t.count = 0;
  __syncthreads();
  if (tid >= 192) {
    const uint32_t b = a.K > 0 ? bound_of<256>(t.maxima, a.K, lane) : 0;
    if (lane == 0) t.bound = b;
  }
  if (tid < 64) {
    Sums x{-INFINITY, 0.f, 0.f};
    for (int i = lane; i < segs; i += 64) {
      const float4 p = out.part[row * segs + i];
      add(x, Sums{p.x, p.y, p.z}, c);
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      // the lower lane's first, in both: the same sum in the same order
      const Sums y{__shfl_xor(x.m, off, 64), __shfl_xor(x.s, off, 64), __shfl_xor(x.u, off, 64)};
      Sums lower = lane & off ? y : x;
      add(lower, lane & off ? x : y, c);
      x = lower;
    }
    if (lane == 0) {
      all = x;
      row_result<T>(a, row, x, out.logp, out.entropy, out.stats);
    }
  }
  __syncthreads();
  if (a.K == 0) return;
  const uint64_t bound = (uint64_t)t.bound << 32;
  for (int i = tid; i < total; i += 256) {
    const uint64_t p = pairs[i];
    if (p >= bound && p != 0) {
      const int at = atomicAdd(&t.count, 1);
      if (at < kMost) t.found[0][at] = p;
    }
  }
  __syncthreads();
  int n = t.count;
  if (n > kMost) {  // many equal logits: pairs differ all the same
    uint64_t lo = bound, hi = ~0ull;
    int turn = 0;
    while (n > kMost) {
      const uint64_t mid = lo + (hi - lo) / 2;
      int k = 0;
      for (int i = tid; i < total; i += 256) k += pairs[i] >= mid && pairs[i] != 0;
      k = count_all(t, k, turn++);
      if (k >= a.K)
        lo = mid, n = k;
      else
        hi = mid;
    }
    __syncthreads();
    if (tid == 0) t.count = 0;
    __syncthreads();
    for (int i = tid; i < total; i += 256) {
      const uint64_t p = pairs[i];
      if (p >= lo && p != 0) {
        const int at = atomicAdd(&t.count, 1);
        if (at < kMost) t.found[0][at] = p;
      }
    }
    __syncthreads();
    n = min(t.count, kMost);
  }
  const Result r(all, a.tau);
  rank_top<256>(t.found[0], n, a.K, [&](int rank, uint64_t pair) {
    out.idx[row * a.K + rank] = place_of(pair);
    out.top[row * a.K + rank] = r.logp(of_key((uint32_t)(pair >> 32)));
  });
}

// ---- gradient ------------------------------------------------------------------
constexpr int kGradThreads = 256;

// Segment blockIdx.x of a row of the gradient.  z and gz may be the same memory: a thread reads the logits it
// writes the gradients of, and the named places' are read before.
template <class T>
__global__ __launch_bounds__(kGradThreads) void k_logprobs_grad(fdc_token_logprobs_args a, const float *__restrict__ stats,
                                                                const float *__restrict__ glogp,
                                                                const float *__restrict__ gentropy,
                                                                const int32_t *__restrict__ idx,
                                                                const float *__restrict__ gtop, void *gz_,
                                                                int64_t gz_stride, int seg) {
  constexpr int V = kLogitV<T>;
  __shared__ int place[kLogprobMaxTop + 1];
  __shared__ float target[kLogprobMaxTop + 1], logit[kLogprobMaxTop + 1];
  const int64_t row = (int64_t)blockIdx.y + (int64_t)blockIdx.z * 32768;
  if (row >= a.R) return;
  const int tid = threadIdx.x, K = gtop != nullptr ? a.K : 0;
  const T *z = static_cast<const T *>(a.z) + row * a.z_stride;
  T *gz = static_cast<T *>(gz_) + row * gz_stride;
  // entry 0 is the token
  for (int k = tid; k <= K; k += kGradThreads) {
    const int v = k == 0 ? (glogp != nullptr ? a.tokens[row] : -1) : idx[row * a.K + k - 1];
    place[k] = v;
    target[k] = v < 0 ? 0.f : k == 0 ? glogp[row] : gtop[row * a.K + k - 1];
    logit[k] = v >= 0 && v < a.V ? (float)z[v] : 0.f;
  }
  __syncthreads();
  // every wave for itself: the entries' sum, and whether one is not 0, or names a place past the vocabulary
  float alike = 0.f;
  int flags = 0;
  for (int k = tid & 63; k <= K; k += 64) {
    alike += target[k];
    flags |= (target[k] != 0.f ? 1 : 0) | (place[k] >= a.V ? 2 : 0);
  }
  alike = wave_sum(alike);
  const bool any = __any(flags & 1), over = __any(flags & 2);
  const float gh = gentropy != nullptr ? gentropy[row] : 0.f;
  const int begin = blockIdx.x * seg, end = min(a.V, begin + seg);
  if (!any && gh == 0.f) {
    const float o[V] = {};
    for (int at = begin + tid * V; at < end; at += kGradThreads * V) store_some<T, V>(gz + at, o, min(V, end - at));
    return;
  }
  const float *p = stats + kLogprobStats * row;
  // 1 / tau as a factor of p where it is large, and of the upstream gradients where it is small: 1 / (tau s) is not among
  // float32's normal numbers at the hottest temperatures, and the gradients over tau are too large at the coldest
  const float per = 1.f / a.tau, c = kLog2e / a.tau, m = p[0], f = over ? NAN : fmaxf(per, 1.f) / p[1], g = fminf(per, 1.f);
  // p (l + entropy) with l = t log(2) - log s, t = (z - m) log2(e) / tau
  const float shift = p[2] - __builtin_amdgcn_logf(p[1]) * kLn2;
  const float c0 = fmaf(gh, shift, alike) * g, c1 = gh * kLn2 * g;
  auto grad = [&](float x) {
    const float t = (x - m) * c;
    return -f * exp2_fast(t) * fmaf(c1, fmaxf(t, -300.f), c0);  // past -300 the exponential is 0, and its factor finite
  };
  for (int at = begin + tid * V; at < end; at += kGradThreads * V) {
    const int n = min(V, end - at);
    const Pack<T, V> x = load_some<T, V>(z + at, n);
    float o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = grad(x.at(i));
    store_some<T, V>(gz + at, o, n);
  }
  __syncthreads();
  // the named places: the first entry of a place adds all of its targets
  for (int k = tid; k <= K; k += kGradThreads) {
    const int v = place[k];
    if (v < begin || v >= end) continue;
    float sum = 0.f;
    bool first = true;
    for (int j = 0; j <= K; ++j) {
      const bool same = place[j] == v;
      sum += same ? target[j] : 0.f;
      first = first && !(same && j < k);
    }
    if (first) gz[v] = (T)(fmaf(sum, per, grad(logit[k])));
  }
}

// ---- host ----------------------------------------------------------------------
struct Segments {
  int seg, segs;
  bool wide;
};
constexpr int kThreads = 256, kManyThreads = 1024, kPieces = 4;  // of a chunk
// A row a workgroup where there are rows for every compute unit, and for fewer ones of at most 256 KB, in workgroups of 1024
// threads (one launch without a workspace instead of two); else segments of one chunk or more.  A call with 20 best in one
// launch and in segments, in a captured graph, us: 32000 bf16 (64 KB), 1 row 9.7 and 11.1, 64 rows 11.5 and 14.5, 500 rows 16.9
// and 23.4; 50021 f32 (200 KB) 15.9 and 10.4, 16.9 and 12.4, 28.8 and 32.8; 128256 bf16 (250 KB) 22.1 and 11.8, 24.6 and 17.7,
// 41.2 and 51.4; 151936 bf16 (297 KB) 26.1 and 11.7, 28.8 and 18.9, 48.6 and 55.5.  So up to 64 rows of more than some 80 KB
// would be better off in segments, and 500 of any size here in one launch.
Segments segments(int dtype, int64_t R, int V) {
  const int piece = 16 / (int)dtype_size(dtype), chunk = kThreads * kPieces * piece;
  const long long chunks = ceil_div(V, chunk);
  long long per = std::max(1LL, std::min<long long>(chunks, R * chunks / 1024));  // chunks a segment
  Segments s;
  s.wide = per < chunks && V * (long long)dtype_size(dtype) <= 256 << 10;
  if (s.wide) per = chunks;
  s.seg = (int)(per * chunk);
  s.segs = (int)ceil_div(V, s.seg);
  return s;
}
Segments grad_segments(int dtype, int64_t R, int V) {
  const int unit = kGradThreads * 16 / (int)dtype_size(dtype);
  long long per = ceil_div(V, unit);
  while (per > 1 && R * ceil_div(V, per * unit) < 2048) per = ceil_div(per, 2);
  Segments s{};
  s.seg = (int)(per * unit);
  s.segs = (int)ceil_div(V, s.seg);
  return s;
}
dim3 wide_grid(long long n) { return dim3((unsigned)std::min<long long>(n, 32768), (unsigned)ceil_div(n, 32768)); }

// f(threads, pieces a thread) of a chunk, for segments of `vecs` 16-byte pieces.
template <class F>
hipError_t by_pieces(long long vecs, bool wide, F &&f) {
  using std::integral_constant;
  if (wide) return f(integral_constant<int, kManyThreads>{}, integral_constant<int, kPieces>{});
  if (vecs <= 64) return f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (vecs <= kThreads) return f(integral_constant<int, kThreads>{}, integral_constant<int, 1>{});
  return f(integral_constant<int, kThreads>{}, integral_constant<int, kPieces>{});
}

}  // namespace

size_t token_logprobs_ws(int dtype, int64_t R, int V, int K) {
  const Segments sg = segments(dtype, R, V);
  return sg.segs == 1 ? 0 : (size_t)R * sg.segs * (sizeof(float4) + K * sizeof(uint64_t));
}

hipError_t launch_token_logprobs(const fdc_token_logprobs_args &a, float *logp, float *entropy, int32_t *idx, float *top,
                                 float *stats, void *ws, hipStream_t s) {
  const Segments sg = segments(a.dtype, a.R, a.V);
  float4 *part = static_cast<float4 *>(ws);
  const Out out{logp, entropy, idx, top, stats, part, reinterpret_cast<uint64_t *>(part + a.R * sg.segs)};
  return by_dtype(a.dtype, [&](auto tag) {
    using T = decltype(tag);
    if (hipError_t e = by_pieces(ceil_div(std::min(sg.seg, a.V), kLogitV<T>), sg.wide, [&](auto threads, auto pieces) {
          constexpr int TH = decltype(threads)::value, NV = decltype(pieces)::value;
          return timed_launch("logprobs", a.K > 0 ? k_logprobs<T, TH, NV, true> : k_logprobs<T, TH, NV, false>,
                              wide_grid(a.R * sg.segs), dim3(TH), 0, s, a, out, sg.seg, sg.segs);
        }))
      return e;
    if (sg.segs == 1) return hipSuccess;
    return timed_launch("logprobs_join", k_logprobs_join<T>, wide_grid(a.R), dim3(256), 0, s, a, out, sg.segs);
  });
}

hipError_t launch_token_logprobs_bwd(const fdc_token_logprobs_args &a, const float *stats, const float *glogp,
                                     const float *gentropy, const int32_t *idx, const float *gtop, void *gz,
                                     int64_t gz_stride, hipStream_t s) {
  const Segments sg = grad_segments(a.dtype, a.R, a.V);
  const dim3 grid((unsigned)sg.segs, (unsigned)std::min<int64_t>(a.R, 32768), (unsigned)ceil_div(a.R, 32768));
  return by_dtype(a.dtype, [&](auto tag) {
    return timed_launch("logprobs_grad", k_logprobs_grad<decltype(tag)>, grid, dim3(kGradThreads), 0, s, a, stats, glogp,
                        gentropy, idx, gtop, gz, gz_stride, sg.seg);
  });
}

}  // namespace fdc
