// Selective state space scan of each channel, its backward, and its form for one token.
//
//   delta = softplus(dt + dt_bias);  h[t][n] = exp(delta A[n]) h[t-1][n] + delta x B[t][n]
//   y[t] = (sum_n C[t][n] h[t][n] + skip x) silu(gate)
//
// Backward, with gs = gy silu(gate), u = delta x and the adjoint of h[t]
//   g[t][n] = exp(delta[t+1] A[n]) g[t+1][n] + C[t][n] gs[t]:
//   gB[t][n] = sum_d g u;  gC[t][n] = sum_d h gs;  gu = sum_n g B;  e[n] = g exp(delta A) h[t-1]
//   gdelta = sum_n e A + gu x;  gx = gu delta + gs skip;  gA = sum_t e delta.
//
// The decay differs for every channel, state and token, so there is no matrix product in it: each
// (token, channel, state) takes an exponential (four issue slots of a full-rate operation) and
// four multiplications and additions forward, about thirteen backward.  The vector units bound both;
// HBM would take a ninth of the time (8 x 1024 tokens, 2048 channels of 16 states, bf16: 143 us
// forward, 348 us backward; one sequence of 16384 tokens: 259 us forward).  Counted at 8 x 1024 tokens:
// the vector units are busy for 85 and 88 % of the forward passes' cycles, with 8.3 and 5.5 instructions a
// state and token, and for 78 and 76 % of the backward ones', with 6.2 and 25; LDS for 30 % of the
// backward's (the channel sums of gB and gC), without bank conflicts.
//
// LN adjacent lanes share a channel and hold SN = 4 states each, so a wave owns 64 / LN channels and
// walks along the tokens in blocks of 16.  What a token needs once per channel (softplus, gate,
// loads and stores) is spread over the LN lanes: lane q of a channel does it for the tokens q,
// q + LN, ... of the block, and the values are handed round with lane moves.  B and C of a block go
// through LDS as floats, shared by the workgroup's channels.
//
// Where the channels of the batch are too few waves for the chip, the tokens are cut into chunks: a
// first pass finds what each chunk adds to a zero state and how much it decays one, a small second
// one carries the states over the chunks, and the scan proper runs on every chunk at once.
#include <algorithm>

#include "sequence.h"

namespace fdc {

constexpr int kTok = kScanBlock;
constexpr int SN = 4;          // states a lane
constexpr int kScanWaves = 4;  // waves of a workgroup, side by side in the channels

struct ScanGrid {
  int Dg;      // channels a group
  int tiles;   // workgroups a group
  int chunk;   // tokens a chunk (a multiple of kTok)
  int chunks;  // chunks a sequence
  int blocks;  // saved states a sequence: ceil(L / kTok)
};

template <int LN>
struct ScanLane {
  static constexpr int NP = SN * LN;          // states, padded
  static constexpr int CW = 64 / LN;          // channels a wave
  static constexpr int Waves = kScanWaves, Threads = 64 * Waves;
  static constexpr int CG = CW * Waves;       // channels a workgroup
  static constexpr int E = kTok / LN;         // tokens of a block a lane does the channel's work for
  int q, g, d, nvalid;                        // lane of the channel; group; channel; states here
  bool live, full;                            // the channel is there; all of the workgroup's are
  __device__ __forceinline__ ScanLane(const ScanGrid &sg, int N) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    q = lane % LN;
    g = blockIdx.x / sg.tiles;
    const int ch = (blockIdx.x - g * sg.tiles) * CG + wave * CW + lane / LN;
    live = ch < sg.Dg;
    full = (int)(blockIdx.x - g * sg.tiles + 1) * CG <= sg.Dg;
    d = g * sg.Dg + ch;
    nvalid = live ? max(0, min(SN, N - SN * q)) : 0;
  }
};

// The states of a [.][N] float row that a lane holds, those that are there.
__device__ __forceinline__ void load_states(float (&v)[SN], const float *p, int nvalid) {
#pragma unroll
  for (int r = 0; r < SN; ++r) v[r] = 0.f;
  if (nvalid > 0) {
    const Pack<float, SN> x = load_some<float, SN>(p, nvalid);
#pragma unroll
    for (int r = 0; r < SN; ++r) v[r] = x.at(r);
  }
}
__device__ __forceinline__ void store_states(float *p, const float (&v)[SN], int nvalid) {
  if (nvalid > 0) store_some<float, SN>(p, v, nvalid);
}
__device__ __forceinline__ void read_lds(float (&v)[SN], const float *p) {
  const float4 x = *reinterpret_cast<const float4 *>(p);
  v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
}
__device__ __forceinline__ void write_lds(float *p, const float (&v)[SN]) {
  *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
}

// a and b summed over lane pairs at distance M (1 or 2): the lane with bit M clear gets a's sum, the other b's.
template <int M>
__device__ __forceinline__ float pair_sum(float a, float b, int q) {
  const bool up = q & M;
  const float keep = up ? b : a, send = up ? a : b;
  return keep + dpp<M == 1 ? 0xB1 : 0x4E>(send);
}
// Sums over a channel's LN lanes of four tokens' values s (tokens Base .. Base + 3 of the block), each
// to the lane that stands for its token.
template <int LN, int Base, int E>
__device__ __forceinline__ void token_sums(const float (&s)[4], float (&dst)[E], int q) {
  const float lo = pair_sum<1>(s[0], s[1], q), hi = pair_sum<1>(s[2], s[3], q);
  if constexpr (LN == 2) {
    dst[Base / 2] = lo;
    dst[Base / 2 + 1] = hi;
  } else {
    float v = pair_sum<2>(lo, hi, q);
    if constexpr (LN >= 8) v += dpp<0x141>(dpp<0x1B>(v));  // lane ^ 3, then mirrored in 8: lane ^ 4
    if constexpr (LN >= 16) v += dpp<0x128>(v);            // turned by 8 in 16: lane ^ 8
    dst[Base / LN] = LN == 4 || q / 4 == Base % LN / 4 ? v : dst[Base / LN];
  }
}

// A [L][width] tensor of one sequence at the block of tokens that is being worked on.  Base and stride are
// the same in every lane, so that an access is a scalar base and a 32-bit offset of the lane in bytes
// (token strides are below 2^25 elements, columns below 2^20).
template <class T>
struct Rows {
  char *p;
  int stride;  // bytes
  __device__ __forceinline__ Rows(const fdc_tokens &t, int b, int t0, int64_t column = 0)
      : p(reinterpret_cast<char *>(static_cast<T *>(t.p) + (t.p ? b * t.batch_stride + t0 * t.token_stride + column : 0))),
        stride((int)t.token_stride * (int)sizeof(T)) {}
  __device__ __forceinline__ unsigned offset(int s, int column) const {
    return (unsigned)s * (unsigned)stride + (unsigned)column * (unsigned)sizeof(T);
  }
  __device__ __forceinline__ T &at(unsigned off) const { return *reinterpret_cast<T *>(p + off); }
  __device__ __forceinline__ void next() { p += (int64_t)stride * kTok; }
  __device__ __forceinline__ void previous() { p -= (int64_t)stride * kTok; }
};

// B and C of a block of tokens: each thread's share of the loads, and its way into LDS
// ([kTok][NP] floats each; zero for padded states and for tokens from `len` on).
template <class T, int LN, bool WithC>
struct BlockBC {
  static constexpr int NP = ScanLane<LN>::NP, Threads = ScanLane<LN>::Threads;
  static constexpr int Per = (kTok * NP + Threads - 1) / Threads;
  T b[Per], c[Per];
  // t0 < L; tokens past L are read as the last one
  __device__ __forceinline__ void load(const Rows<T> &B, const Rows<T> &C, int t0, int L, int N) {
#pragma unroll
    for (int k = 0; k < Per; ++k) {
      const int i = threadIdx.x + k * Threads, s = min(min(i / NP, kTok - 1), L - 1 - t0), n = min(i % NP, N - 1);
      b[k] = B.at(B.offset(s, n));
      if constexpr (WithC) c[k] = C.at(C.offset(s, n));
    }
  }
  __device__ __forceinline__ void put(float *Bs, float *Cs, int t0, int len, int N) const {
#pragma unroll
    for (int k = 0; k < Per; ++k) {
      const int i = threadIdx.x + k * Threads;
      const bool in = t0 + i / NP < len && i % NP < N;
      if (Per * Threads == kTok * NP || i < kTok * NP) {
        Bs[i] = in ? (float)b[k] : 0.f;
        if constexpr (WithC) Cs[i] = in ? (float)c[k] : 0.f;
      }
    }
  }
};

// One lane's values of a [L][D] tensor at its tokens of a block, as they lie in memory: those of tokens
// and channels that are not there are another's and have to be left out.
template <class T, int LN>
struct LaneTokens {
  static constexpr int E = kTok / LN;
  T v[E];
  __device__ __forceinline__ void load(const Rows<T> &r, int t0, int q, int dc, int L) {
    if (t0 + kTok <= L) {
      const unsigned off = r.offset(q, dc);
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = r.at(off + (unsigned)(i * LN) * (unsigned)r.stride);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = r.at(r.offset(min(i * LN + q, L - 1 - t0), dc));
    }
  }
};
// Stores of a lane's tokens of a block below `end` (exclusive), by the lanes whose channel is there.
template <class T, int LN, int E>
__device__ __forceinline__ void store_tokens(const Rows<T> &r, const float (&v)[E], int t0, int q, int dc, int end,
                                             bool live) {
  if (!live) return;
  const unsigned off = r.offset(q, dc);
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (t0 + i * LN + q < end) r.at(off + (unsigned)(i * LN) * (unsigned)r.stride) = (T)v[i];
}

// Formed for every lane, there or not, so that the block's tokens go through it side by side.
__device__ __forceinline__ float step_size(float raw, int use_softplus, bool in) {
  const float v = softplus(raw);
  return in ? (use_softplus ? v : raw) : 0.f;
}

// Local: the chunk from a zero state, without outputs: its last state goes to
// carry [B][chunks][D][N], the sum of delta to dsum [B][chunks][D].  Otherwise the scan proper,
// from h0 (one chunk) or carry.
template <class T, int LN, bool Local>
__global__ __launch_bounds__(ScanLane<LN>::Threads) void k_scan_fwd(fdc_scan_args a, ScanGrid sg, float *__restrict__ carry,
                                                              float *__restrict__ dsum, float *__restrict__ saved) {
  using Lane = ScanLane<LN>;
  constexpr int NP = Lane::NP, E = Lane::E;
  __shared__ __align__(16) float Bs[2][kTok * NP], Cs[Local ? 1 : 2][Local ? 4 : kTok * NP];
  const Lane ln(sg, a.N);
  const int b = blockIdx.z, chunk = blockIdx.y;
  const int len = length_of(a.lengths, b, a.L);
  const int t_begin = chunk * sg.chunk, t_end = min(a.L, t_begin + sg.chunk);
  const int dc = ln.live ? ln.d : 0;  // a channel whose address exists
  Rows<T> xr(a.x, b, t_begin), dtr(a.dt, b, t_begin), gr(a.gate, b, t_begin), yr(a.y, b, t_begin);
  Rows<T> Br(a.Bm, b, t_begin, ln.g * a.N), Cr(a.Cm, b, t_begin, ln.g * a.N);
  const bool gated = !Local && a.gate.p != nullptr;
  const float bias = a.dt_bias && ln.live ? a.dt_bias[dc] : 0.f, skip = a.skip && ln.live ? a.skip[dc] : 0.f;

  float A2[SN], h[SN];
  load_states(A2, a.A + (int64_t)dc * a.N + SN * ln.q, ln.nvalid);
#pragma unroll
  for (int r = 0; r < SN; ++r) A2[r] *= kLog2e;
  const int64_t state_at = ((int64_t)b * a.D + dc) * a.N + SN * ln.q;
  const int64_t carry_at = (((int64_t)b * sg.chunks + chunk) * a.D + dc) * a.N + SN * ln.q;
#pragma unroll
  for (int r = 0; r < SN; ++r) h[r] = 0.f;
  if constexpr (!Local) {
    if (sg.chunks > 1)
      load_states(h, carry + carry_at, ln.nvalid);
    else if (a.h0)
      load_states(h, a.h0 + state_at, ln.nvalid);
  }
  float dtotal = 0.f;

  BlockBC<T, LN, !Local> bc;
  LaneTokens<T, LN> tx, tdt, tg;
  auto fetch = [&](int t0) {
    bc.load(Br, Cr, t0, a.L, a.N);
    tx.load(xr, t0, ln.q, dc, a.L);
    tdt.load(dtr, t0, ln.q, dc, a.L);
    if (gated) tg.load(gr, t0, ln.q, dc, a.L);
    xr.next(), dtr.next(), gr.next(), Br.next(), Cr.next();
  };
  fetch(t_begin);
  float *sp = saved ? saved + (((int64_t)b * sg.blocks + t_begin / kTok) * a.D + dc) * a.N + SN * ln.q : nullptr;
  for (int t0 = t_begin, it = 0; t0 < t_end; t0 += kTok, it ^= 1) {
    float delta[E], u[E], x[E], gate[E], out[E];
    bc.put(Bs[it], Cs[Local ? 0 : it], t0, len, a.N);
    auto begin_tokens = [&](auto whole) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const bool in = whole.value || (ln.live && t0 + i * LN + ln.q < len);
        x[i] = in ? (float)tx.v[i] : 0.f;
        gate[i] = gated ? (float)tg.v[i] : 0.f;
        delta[i] = step_size((float)tdt.v[i] + bias, a.softplus, in);
        u[i] = delta[i] * x[i];
        out[i] = 0.f;
        dtotal += delta[i];
      }
    };
    if (ln.full && t0 + kTok <= len)
      begin_tokens(std::true_type{});
    else
      begin_tokens(std::false_type{});
    __syncthreads();
    if (t0 + kTok < t_end) fetch(t0 + kTok);
    if constexpr (!Local)
      if (saved) {
        store_states(sp, h, ln.nvalid);
        sp += (int64_t)a.D * a.N;
      }
    if (t0 < len) {
      static_for<kTok / 4>([&](auto four) {
        constexpr int Base = 4 * decltype(four)::value;
        float sums[4];
        static_for<4>([&](auto step) {
          constexpr int K = decltype(step)::value, S = Base + K, i = S / LN, src = S % LN;
          const float dl = lane_bcast<LN, src>(delta[i]), us = lane_bcast<LN, src>(u[i]);
          float Bq[SN];
          read_lds(Bq, &Bs[it][S * NP + SN * ln.q]);
#pragma unroll
          for (int r = 0; r < SN; ++r) h[r] = fmaf(exp2_fast(dl * A2[r]), h[r], us * Bq[r]);
          if constexpr (!Local) {
            float Cq[SN];
            read_lds(Cq, &Cs[it][S * NP + SN * ln.q]);
            sums[K] = Cq[0] * h[0];
#pragma unroll
            for (int r = 1; r < SN; ++r) sums[K] = fmaf(Cq[r], h[r], sums[K]);
          }
        });
        if constexpr (!Local) token_sums<LN, Base, E>(sums, out, ln.q);
      });
    }
    if constexpr (!Local) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        out[i] = fmaf(skip, x[i], out[i]);
        if (gated) out[i] *= gate[i] * sigmoid(gate[i]);
        if (t0 + i * LN + ln.q >= len) out[i] = 0.f;
      }
      store_tokens<T, LN>(yr, out, t0, ln.q, dc, t_end, ln.live);
      yr.next();
    }
  }
  if constexpr (Local) {
    store_states(carry + carry_at, h, ln.nvalid);
    dtotal = lane_sum<LN>(dtotal);
    if (ln.live && ln.q == 0) dsum[((int64_t)b * sg.chunks + chunk) * a.D + ln.d] = dtotal;
  } else if (a.h_last && t_end == a.L) {
    store_states(a.h_last + state_at, h, ln.nvalid);
  }
}

// carry [B][chunks][D][N], what each chunk adds to a zero state, becomes the state that each chunk starts
// from: a thread a (sequence, channel, state), over the chunks in order (the adjoint: from the last).
__global__ __launch_bounds__(256) void k_scan_carry(float *__restrict__ carry, const float *__restrict__ dsum,
                                                    const float *__restrict__ A, const float *__restrict__ h0, int B,
                                                    int D, int N, int chunks, int reverse) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, DN = (int64_t)D * N;
  if (i >= B * DN) return;
  const int64_t b = i / DN, dn = i - b * DN, d = dn / N;
  const float A2 = A[dn] * kLog2e;
  float h = h0 ? h0[i] : 0.f;
  constexpr int Ahead = 8;  // chunks loaded together: the loop is bound by their latency
  for (int k0 = 0; k0 < chunks; k0 += Ahead) {
    float local[Ahead], total[Ahead];
#pragma unroll
    for (int u = 0; u < Ahead; ++u) {
      const int k = min(k0 + u, chunks - 1);
      const int64_t c = b * chunks + (reverse ? chunks - 1 - k : k);
      local[u] = carry[c * DN + dn];
      total[u] = dsum[c * D + d];
    }
#pragma unroll
    for (int u = 0; u < Ahead; ++u) {
      const int k = k0 + u;
      if (k >= chunks) break;
      const int64_t c = b * chunks + (reverse ? chunks - 1 - k : k);
      carry[c * DN + dn] = h;
      h = fmaf(exp2_fast(A2 * total[u]), h, local[u]);
    }
  }
}

// The adjoint of a chunk from a zero one behind it: what reaches the state in front of the chunk.
template <class T, int LN>
__global__ __launch_bounds__(ScanLane<LN>::Threads) void k_scan_bwd_local(fdc_scan_args a, fdc_tokens gy, ScanGrid sg,
                                                                    float *__restrict__ carry,
                                                                    float *__restrict__ dsum) {
  using Lane = ScanLane<LN>;
  constexpr int NP = Lane::NP, E = Lane::E;
  __shared__ __align__(16) float Cs[2][kTok * NP];
  const Lane ln(sg, a.N);
  const int b = blockIdx.z, chunk = blockIdx.y;
  const int len = length_of(a.lengths, b, a.L);
  const int t_begin = chunk * sg.chunk, t_end = min(a.L, t_begin + sg.chunk);
  const int dc = ln.live ? ln.d : 0;
  const int t_last = t_begin + (t_end - t_begin - 1) / kTok * kTok;
  Rows<T> dtr(a.dt, b, t_last), gyr(gy, b, t_last), gr(a.gate, b, t_last), Cr(a.Cm, b, t_last, ln.g * a.N);
  const bool gated = a.gate.p != nullptr;
  const float bias = a.dt_bias && ln.live ? a.dt_bias[dc] : 0.f;
  float A2[SN], g[SN];
  load_states(A2, a.A + (int64_t)dc * a.N + SN * ln.q, ln.nvalid);
#pragma unroll
  for (int r = 0; r < SN; ++r) {
    A2[r] *= kLog2e;
    g[r] = 0.f;
  }
  float dtotal = 0.f;
  BlockBC<T, LN, false> cc;
  LaneTokens<T, LN> tdt, tgy, tg;
  auto fetch = [&](int t0) {
    cc.load(Cr, Cr, t0, a.L, a.N);
    tdt.load(dtr, t0, ln.q, dc, a.L);
    tgy.load(gyr, t0, ln.q, dc, a.L);
    if (gated) tg.load(gr, t0, ln.q, dc, a.L);
    dtr.previous(), gyr.previous(), gr.previous(), Cr.previous();
  };
  fetch(t_last);
  for (int t0 = t_last, it = 0; t0 >= t_begin; t0 -= kTok, it ^= 1) {
    float delta[E], gs[E];
    cc.put(Cs[it], nullptr, t0, len, a.N);
    auto begin_tokens = [&](auto whole) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const bool in = whole.value || (ln.live && t0 + i * LN + ln.q < len);
        const float gate = gated ? (float)tg.v[i] : 0.f;
        delta[i] = step_size((float)tdt.v[i] + bias, a.softplus, in);
        gs[i] = (float)tgy.v[i];
        if (gated) gs[i] *= gate * sigmoid(gate);
        if (!in) gs[i] = 0.f;
        dtotal += delta[i];
      }
    };
    if (ln.full && t0 + kTok <= len)
      begin_tokens(std::true_type{});
    else
      begin_tokens(std::false_type{});
    __syncthreads();
    if (t0 > t_begin) fetch(t0 - kTok);
    if (t0 < len) {
      static_for<kTok>([&](auto step) {
        constexpr int S = kTok - 1 - decltype(step)::value, i = S / LN, src = S % LN;
        const float dl = lane_bcast<LN, src>(delta[i]), gss = lane_bcast<LN, src>(gs[i]);
        float Cq[SN];
        read_lds(Cq, &Cs[it][S * NP + SN * ln.q]);
#pragma unroll
        for (int r = 0; r < SN; ++r) g[r] = exp2_fast(dl * A2[r]) * fmaf(Cq[r], gss, g[r]);
      });
    }
  }
  store_states(carry + (((int64_t)b * sg.chunks + chunk) * a.D + dc) * a.N + SN * ln.q, g, ln.nvalid);
  dtotal = lane_sum<LN>(dtotal);
  if (ln.live && ln.q == 0) dsum[((int64_t)b * sg.chunks + chunk) * a.D + ln.d] = dtotal;
}

// The backward proper.  A block's states are formed again from the saved one in front of it and
// kept in registers (16 tokens x 4 states), then the block is walked backwards, with each decay formed
// once more.  Two waves a SIMD by its registers: with four lanes a channel (9 to 16 states) the bound of
// 256 spills 4 of them in 16 bits and 19 in float32; with two (up to 8 states) a bound of two waves would
// spill far more, and one wave a SIMD is left.
// The sums of gB and gC over the channels: every fourth token the lanes put their four products of
// four tokens into LDS and add them up over the wave's channels the other way round; the waves'
// sums are added in wave order, and the workgroups' partial sums
// (partBC [2][tiles][B][L][G N]) by k_scan_sum_bc.  partP [B chunks][D N + 2 D]: gA, gskip, gdt_bias.
template <class T, int LN>
__global__ __launch_bounds__(ScanLane<LN>::Threads, LN == 2 ? 1 : 2) void k_scan_bwd(fdc_scan_args a, fdc_scan_grads gr, ScanGrid sg,
                                                              const float *__restrict__ saved,
                                                              const float *__restrict__ carry,
                                                              float *__restrict__ partBC,
                                                              float *__restrict__ partP) {
  using Lane = ScanLane<LN>;
  constexpr int NP = Lane::NP, E = Lane::E, CW = Lane::CW;
  constexpr int kSteps = 4;                   // tokens a round of the channel sums takes
  constexpr int Row = 64 * SN + 16;           // floats of one (token, kind): the lanes' states, and a shift of banks
  constexpr int Outs = kSteps * 2 * LN;       // sums (of SN states each) a round forms
  constexpr int Parts = Outs < 64 ? 64 / Outs : 1;  // lanes that share one
  constexpr int Rounds = Outs < 64 ? 1 : Outs / 64;
  constexpr int Sum = CW / Parts;             // channels a lane adds
  __shared__ __align__(16) float Bs[kTok * NP], Cs[kTok * NP];
  __shared__ __align__(16) float prod[Lane::Waves][kSteps * 2 * Row];
  __shared__ __align__(16) float wsum[Lane::Waves][kTok * 2 * NP];
  const Lane ln(sg, a.N);
  const int b = blockIdx.z, chunk = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int len = length_of(a.lengths, b, a.L);
  const int t_begin = chunk * sg.chunk, t_end = min(a.L, t_begin + sg.chunk);
  const int dc = ln.live ? ln.d : 0;
  const int t_last = t_begin + (t_end - t_begin - 1) / kTok * kTok;
  Rows<T> xr(a.x, b, t_last), dtr(a.dt, b, t_last), gyr(gr.gy, b, t_last), gtr(a.gate, b, t_last);
  Rows<T> Br(a.Bm, b, t_last, ln.g * a.N), Cr(a.Cm, b, t_last, ln.g * a.N);
  Rows<T> gxr(gr.gx, b, t_last), gdtr(gr.gdt, b, t_last), ggr(gr.ggate, b, t_last);
  const bool gated = a.gate.p != nullptr;
  const float bias = a.dt_bias && ln.live ? a.dt_bias[dc] : 0.f, skip = a.skip && ln.live ? a.skip[dc] : 0.f;
  const int tile = blockIdx.x - ln.g * sg.tiles;
  const int64_t GN = (int64_t)a.G * a.N, kind_stride = (int64_t)sg.tiles * a.B * a.L * GN;
  float *pbc = partBC + ((int64_t)tile * a.B + b) * a.L * GN + ln.g * a.N;

  float A2[SN], g[SN], gA[SN], gskip = 0.f, gbias = 0.f;
  load_states(A2, a.A + (int64_t)dc * a.N + SN * ln.q, ln.nvalid);
#pragma unroll
  for (int r = 0; r < SN; ++r) {
    A2[r] *= kLog2e;
    g[r] = gA[r] = 0.f;
  }
  if (sg.chunks > 1) load_states(g, carry + (((int64_t)b * sg.chunks + chunk) * a.D + dc) * a.N + SN * ln.q, ln.nvalid);

  BlockBC<T, LN, true> bc;
  LaneTokens<T, LN> tx, tdt, tg, tgy;
  float hs[SN];
  const float *sp = saved + (((int64_t)b * sg.blocks + t_last / kTok) * a.D + dc) * a.N + SN * ln.q;
  auto fetch = [&](int t0) {
    bc.load(Br, Cr, t0, a.L, a.N);
    tx.load(xr, t0, ln.q, dc, a.L);
    tdt.load(dtr, t0, ln.q, dc, a.L);
    tgy.load(gyr, t0, ln.q, dc, a.L);
    if (gated) tg.load(gtr, t0, ln.q, dc, a.L);
    load_states(hs, sp, ln.nvalid);
    xr.previous(), dtr.previous(), gyr.previous(), gtr.previous(), Br.previous(), Cr.previous();
    sp -= (int64_t)a.D * a.N;
  };
  fetch(t_last);
  for (int t0 = t_last; t0 >= t_begin; t0 -= kTok) {
    float delta[E], u[E], x[E], gs[E], out[E], gu[E], gd[E], gate[E], gyv[E], raw[E];
    bc.put(Bs, Cs, t0, len, a.N);
    float h[kTok + 1][SN];
#pragma unroll
    for (int r = 0; r < SN; ++r) h[0][r] = hs[r];
    auto begin_tokens = [&](auto whole) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const bool in = whole.value || (ln.live && t0 + i * LN + ln.q < len);
        x[i] = in ? (float)tx.v[i] : 0.f;
        gate[i] = in && gated ? (float)tg.v[i] : 0.f;
        gyv[i] = in ? (float)tgy.v[i] : 0.f;
        raw[i] = in ? (float)tdt.v[i] + bias : 0.f;
        delta[i] = step_size(raw[i], a.softplus, in);
        u[i] = delta[i] * x[i];
        gs[i] = gated ? gyv[i] * (gate[i] * sigmoid(gate[i])) : gyv[i];
        out[i] = gu[i] = gd[i] = 0.f;
      }
    };
    if (ln.full && t0 + kTok <= len)
      begin_tokens(std::true_type{});
    else
      begin_tokens(std::false_type{});
    __syncthreads();
    if (t0 > t_begin) fetch(t0 - kTok);
    if (t0 < len) {
      static_for<kTok>([&](auto step) {
        constexpr int S = decltype(step)::value, i = S / LN, src = S % LN;
        const float dl = lane_bcast<LN, src>(delta[i]), us = lane_bcast<LN, src>(u[i]);
        float Bq[SN];
        read_lds(Bq, &Bs[S * NP + SN * ln.q]);
#pragma unroll
        for (int r = 0; r < SN; ++r) {
          h[S + 1][r] = fmaf(exp2_fast(dl * A2[r]), h[S][r], us * Bq[r]);
        }
        if constexpr (S % 4 == 3) __builtin_amdgcn_sched_barrier(0);
      });
      // handed round again on the way back: kept for 16 tokens they would take 32 registers
#pragma unroll
      for (int i = 0; i < E; ++i) asm volatile("" : "+v"(delta[i]), "+v"(u[i]));
      static_for<kTok / kSteps>([&](auto round) {
        constexpr int R = kTok / kSteps - 1 - decltype(round)::value;
        float su[kSteps], sd[kSteps], sy[kSteps];
        static_for<kSteps>([&](auto step) {
          constexpr int K = kSteps - 1 - decltype(step)::value, S = R * kSteps + K, i = S / LN, src = S % LN;
          const float dl = lane_bcast<LN, src>(delta[i]), us = lane_bcast<LN, src>(u[i]);
          const float gss = lane_bcast<LN, src>(gs[i]);
          float Bq[SN], Cq[SN], pB[SN], pC[SN];
          read_lds(Bq, &Bs[S * NP + SN * ln.q]);
          read_lds(Cq, &Cs[S * NP + SN * ln.q]);
          su[K] = sd[K] = sy[K] = 0.f;
#pragma unroll
          for (int r = 0; r < SN; ++r) {
            g[r] = fmaf(Cq[r], gss, g[r]);
            pB[r] = g[r] * us;
            pC[r] = h[S + 1][r] * gss;
            su[K] = fmaf(g[r], Bq[r], su[K]);
            sy[K] = fmaf(Cq[r], h[S + 1][r], sy[K]);
            g[r] *= exp2_fast(dl * A2[r]);
            const float e = g[r] * h[S][r];
            sd[K] = fmaf(e, A2[r], sd[K]);
            gA[r] = fmaf(e, dl, gA[r]);
          }
          float *pw = &prod[wave][K * 2 * Row + SN * lane];
          write_lds(pw, pB);
          write_lds(pw + Row, pC);
        });
        token_sums<LN, R * kSteps, E>(su, gu, ln.q);
        token_sums<LN, R * kSteps, E>(sd, gd, ln.q);
        token_sums<LN, R * kSteps, E>(sy, out, ln.q);
        __builtin_amdgcn_sched_barrier(0);
        wave_sync();
#pragma unroll
        for (int k = 0; k < Rounds; ++k) {
          // this lane's sum: (token, kind) `row`, states SN oq .. SN oq + SN - 1, over `Sum` of the channels
          const int o = (lane + 64 * k) % Outs, row = o / LN, oq = o % LN, first = lane / (Outs < 64 ? Outs : 64) * Sum;
          const float *pr = &prod[wave][row * Row + SN * (first * LN + oq)];
          float s[SN], v[SN];
          read_lds(s, pr);
#pragma unroll
          for (int c = 1; c < Sum; ++c) {
            read_lds(v, pr + SN * c * LN);
#pragma unroll
            for (int r = 0; r < SN; ++r) s[r] += v[r];
          }
#pragma unroll
          for (int off = Outs; off < 64; off <<= 1)
#pragma unroll
            for (int r = 0; r < SN; ++r) s[r] += __shfl_xor(s[r], off, 64);
          if (Parts == 1 || lane < Outs) write_lds(&wsum[wave][(R * kSteps * 2 + row) * NP + SN * oq], s);
        }
        wave_sync();
      });
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const bool in = t0 + i * LN + ln.q < len;
      gd[i] = fmaf(gd[i], kLn2, gu[i] * x[i]);
      if (a.softplus) gd[i] *= sigmoid(raw[i]);
      if (!in) gd[i] = 0.f;
      gskip = fmaf(gs[i], x[i], gskip);
      gbias += gd[i];
      gu[i] = in ? fmaf(gu[i], delta[i], gs[i] * skip) : 0.f;
      if (gated) {
        const float sg_ = sigmoid(gate[i]);
        out[i] = in ? gyv[i] * fmaf(skip, x[i], out[i]) * (sg_ * (1.f + gate[i] * (1.f - sg_))) : 0.f;
      }
    }
    store_tokens<T, LN>(gxr, gu, t0, ln.q, dc, t_end, ln.live);
    store_tokens<T, LN>(gdtr, gd, t0, ln.q, dc, t_end, ln.live);
    if (gated) store_tokens<T, LN>(ggr, out, t0, ln.q, dc, t_end, ln.live);
    gxr.previous(), gdtr.previous(), ggr.previous();
    __syncthreads();
    for (int i = threadIdx.x; i < kTok * 2 * NP; i += Lane::Threads) {
      const int s = i / (2 * NP), kind = i / NP % 2, n = i % NP;
      float v = 0.f;
      if (t0 + s < len)
#pragma unroll
        for (int w = 0; w < Lane::Waves; ++w) v += wsum[w][i];
      if (n < a.N && t0 + s < t_end) pbc[kind * kind_stride + (int64_t)(t0 + s) * GN + n] = v;
    }
  }
  float *pp = partP + ((int64_t)b * sg.chunks + chunk) * ((int64_t)a.D * a.N + 2 * a.D);
  store_states(pp + (int64_t)dc * a.N + SN * ln.q, gA, ln.nvalid);
  gskip = lane_sum<LN>(gskip);
  gbias = lane_sum<LN>(gbias);
  if (ln.live && ln.q == 0) {
    pp[(int64_t)a.D * a.N + ln.d] = gskip;
    pp[(int64_t)a.D * a.N + a.D + ln.d] = gbias;
  }
}

// gB and gC from the workgroups' sums, added in order.
template <class T>
__global__ __launch_bounds__(256) void k_scan_sum_bc(const float *__restrict__ part, fdc_tokens gB, fdc_tokens gC,
                                                     int tiles, int B, int L, int GN) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n = (int64_t)B * L * GN;
  if (i >= n) return;
  const float *p = part + blockIdx.y * (int64_t)tiles * n + i;
  float s = 0.f;
  for (int k = 0; k < tiles; ++k) s += p[k * n];
  const fdc_tokens &o = blockIdx.y ? gC : gB;
  const int64_t bt = i / GN, c = i - bt * GN, b = bt / L, t = bt - b * L;
  static_cast<T *>(o.p)[b * o.batch_stride + t * o.token_stride + c] = (T)s;
}

// One token: LN lanes a channel, for BT sequences, which the channel's parameters are read once for.  A
// pass over the states (HBM: 8 bytes a state): 64 sequences, 4096 channels of 16 states move 34 MB.
template <class T, int LN, int BT>
__global__ __launch_bounds__(256) void k_scan_step(fdc_scan_args a, int Dg) {
  const int i = blockIdx.x * (256 / LN) + threadIdx.x / LN, q = threadIdx.x % LN, b0 = blockIdx.y * BT;
  const bool live = i < a.D;
  const int d = live ? i : 0, g = d / Dg, nvalid = live ? max(0, min(SN, a.N - SN * q)) : 0;
  float A2[SN], h[BT][SN], x[BT], raw[BT], gate[BT];
  Pack<T, SN> Bv[BT], Cv[BT];
#pragma unroll
  for (int k = 0; k < BT; ++k) {
    const int b = min(b0 + k, a.B - 1);
    load_states(h[k], a.h0 + ((int64_t)b * a.D + d) * a.N + SN * q, nvalid);
    x[k] = (float)static_cast<const T *>(a.x.p)[b * a.x.batch_stride + d];
    raw[k] = (float)static_cast<const T *>(a.dt.p)[b * a.dt.batch_stride + d];
    gate[k] = a.gate.p ? (float)static_cast<const T *>(a.gate.p)[b * a.gate.batch_stride + d] : 0.f;
    Bv[k] = Cv[k] = Pack<T, SN>{};
    if (nvalid > 0) {
      Bv[k] = load_some<T, SN>(static_cast<const T *>(a.Bm.p) + b * a.Bm.batch_stride + g * a.N + SN * q, nvalid);
      Cv[k] = load_some<T, SN>(static_cast<const T *>(a.Cm.p) + b * a.Cm.batch_stride + g * a.N + SN * q, nvalid);
    }
  }
  load_states(A2, a.A + (int64_t)d * a.N + SN * q, nvalid);
  const float bias = a.dt_bias ? a.dt_bias[d] : 0.f, skip = a.skip ? a.skip[d] : 0.f;
#pragma unroll
  for (int r = 0; r < SN; ++r) A2[r] *= kLog2e;
#pragma unroll
  for (int k = 0; k < BT; ++k) {
    const int b = b0 + k;
    if (b >= a.B) return;
    const float delta = step_size(raw[k] + bias, a.softplus, true), u = delta * x[k];
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < SN; ++r) {
      h[k][r] = fmaf(exp2_fast(delta * A2[r]), h[k][r], u * Bv[k].at(r));
      s = fmaf(Cv[k].at(r), h[k][r], s);
    }
    store_states(a.h_last + ((int64_t)b * a.D + d) * a.N + SN * q, h[k], nvalid);
    s = fmaf(skip, x[k], lane_sum<LN>(s));
    if (a.gate.p) s *= gate[k] * sigmoid(gate[k]);
    if (live && q == 0) static_cast<T *>(a.y.p)[b * a.y.batch_stride + d] = (T)s;
  }
}

namespace {

int lanes_of(int N) { return N <= 8 ? 2 : N <= 16 ? 4 : N <= 32 ? 8 : 16; }

// One wave on a SIMD issues an instruction every 6.5 cycles, two together every 5, four every 4.5
// (measured), and a chunk's first pass costs about 0.65 of a forward scan and 0.26 of a backward one: the
// forward is cut into chunks where the channels give no more than one wave a SIMD, the backward (two waves
// a SIMD by its registers) where they give fewer than two.  (2048 channels of 16 states, forward:
// 8 x 1024 tokens 163 us whole, 147 us in chunks; 16 x 1024 tokens 204 and 284.  Backward, 8 x 1024
// tokens: 430 us whole, 359 us in chunks.)  The rule was measured at 16 states alone; with up to 8 the
// backward's registers leave it one wave a SIMD whatever the chunks (16 x 1024 tokens: 667 us with 8 states,
// 535 with 16).  The first pass also walks the chunk that none starts from (the forward's last, the backward's
// first), whose result is not used.
// A chunk may be as short as a block; but a block alone takes a wave 3 us forward and 7 us backward and
// the two launches that chunks add 9 us, so that sequences of fewer than 6 and 4 blocks are not cut.
constexpr long long kSimds = 1024;
ScanGrid scan_grid(int B, int L, int D, int N, int G, bool backward) {
  ScanGrid sg;
  sg.Dg = D / G;
  sg.tiles = (int)ceil_div(sg.Dg, 64 / lanes_of(N) * kScanWaves);
  sg.blocks = (int)ceil_div(L, kTok);
  const long long waves = (long long)B * G * sg.tiles * kScanWaves;
  const long long enough = backward ? 2 * kSimds : kSimds + 1, want = backward ? 2 * kSimds : 4 * kSimds;
  const int least = backward ? 4 : 6;
  const long long chunks = waves >= enough || sg.blocks < least ? 1 : std::min<long long>(ceil_div(want, waves), sg.blocks);
  sg.chunk = (int)ceil_div(sg.blocks, chunks) * kTok;
  sg.chunks = (int)ceil_div(L, sg.chunk);
  return sg;
}

size_t round4(size_t n) { return (n + 3) & ~size_t(3); }
size_t carry_floats(const ScanGrid &sg, int B, int D, int N) {
  return sg.chunks > 1 ? round4((size_t)B * sg.chunks * D * N) + round4((size_t)B * sg.chunks * D) : 0;
}

template <class F>
hipError_t by_lanes(int N, F &&f) {
  switch (lanes_of(N)) {
    case 2: return f(std::integral_constant<int, 2>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 8: return f(std::integral_constant<int, 8>{});
    default: return f(std::integral_constant<int, 16>{});
  }
}

hipError_t launch_carry(float *carry, const float *dsum, const float *A, const float *h0, int B, int D, int N,
                        const ScanGrid &sg, int reverse, hipStream_t s) {
  const long long n = (long long)B * D * N;
  return timed_launch("scan_carry", k_scan_carry, dim3((unsigned)ceil_div(n, 256)), dim3(256), 0, s, carry, dsum, A, h0,
                      B, D, N, sg.chunks, reverse);
}

}  // namespace

size_t scan_saved_floats(int B, int L, int D, int N) { return (size_t)B * ceil_div(L, kTok) * D * N; }
size_t scan_fwd_ws_floats(int B, int L, int D, int N, int G) {
  return carry_floats(scan_grid(B, L, D, N, G, false), B, D, N);
}
size_t scan_bwd_ws_floats(int B, int L, int D, int N, int G) {
  const ScanGrid sg = scan_grid(B, L, D, N, G, true);
  return carry_floats(sg, B, D, N) + round4((size_t)B * sg.chunks * ((size_t)D * N + 2 * D)) +
         round4((size_t)2 * sg.tiles * B * L * G * N);
}

hipError_t launch_scan_fwd(const fdc_scan_args &a, float *saved, float *ws, hipStream_t s) {
  const ScanGrid sg = scan_grid(a.B, a.L, a.D, a.N, a.G, false);
  const dim3 grid((unsigned)(a.G * sg.tiles), (unsigned)sg.chunks, (unsigned)a.B), block(64 * kScanWaves);
  float *carry = ws, *dsum = ws ? ws + round4((size_t)a.B * sg.chunks * a.D * a.N) : nullptr;
  return by_dtype(a.dtype, [&](auto tag) {
    using T = decltype(tag);
    return by_lanes(a.N, [&](auto lanes) {
      constexpr int LN = decltype(lanes)::value;
      if (sg.chunks > 1) {
        if (hipError_t e = timed_launch("scan_fwd_local", k_scan_fwd<T, LN, true>, grid, block, 0, s, a, sg, carry, dsum,
                                        (float *)nullptr))
          return e;
        if (hipError_t e = launch_carry(carry, dsum, a.A, a.h0, a.B, a.D, a.N, sg, 0, s)) return e;
      }
      return timed_launch("scan_fwd", k_scan_fwd<T, LN, false>, grid, block, 0, s, a, sg, carry, dsum, saved);
    });
  });
}

hipError_t launch_scan_bwd(const fdc_scan_args &a, const float *saved, const fdc_scan_grads &g, float *ws,
                           hipStream_t s) {
  const ScanGrid sg = scan_grid(a.B, a.L, a.D, a.N, a.G, true);
  const dim3 grid((unsigned)(a.G * sg.tiles), (unsigned)sg.chunks, (unsigned)a.B), block(64 * kScanWaves);
  float *carry = ws, *dsum = ws + round4((size_t)a.B * sg.chunks * a.D * a.N);
  float *partP = ws + carry_floats(sg, a.B, a.D, a.N);
  const long long cols = (long long)a.D * a.N + 2 * a.D, rows = (long long)a.B * sg.chunks;
  float *partBC = partP + round4((size_t)rows * cols);
  const hipError_t e = by_dtype(a.dtype, [&](auto tag) {
    using T = decltype(tag);
    return by_lanes(a.N, [&](auto lanes) {
      constexpr int LN = decltype(lanes)::value;
      if (sg.chunks > 1) {
        if (hipError_t e = timed_launch("scan_bwd_local", k_scan_bwd_local<T, LN>, grid, block, 0, s, a, g.gy, sg, carry,
                                        dsum))
          return e;
        if (hipError_t e = launch_carry(carry, dsum, a.A, nullptr, a.B, a.D, a.N, sg, 1, s)) return e;
      }
      if (hipError_t e = timed_launch("scan_bwd", k_scan_bwd<T, LN>, grid, block, 0, s, a, g, sg, saved, carry, partBC,
                                      partP))
        return e;
      const long long n = (long long)a.B * a.L * a.G * a.N;
      return timed_launch("scan_sum_bc", k_scan_sum_bc<T>, dim3((unsigned)ceil_div(n, 256), 2), dim3(256), 0, s,
                          (const float *)partBC, g.gBm, g.gCm, sg.tiles, a.B, a.L, a.G * a.N);
    });
  });
  if (e != hipSuccess) return e;
  ColSegments segs{};
  segs.count = 3;
  segs.seg[0] = ColSegment{g.gA, a.D * a.N, a.D * a.N, 1};
  segs.seg[1] = ColSegment{g.gskip, a.D, a.D, 1};
  segs.seg[2] = ColSegment{g.gdt_bias, a.D, a.D, 1};
  return launch_col_sums(partP, rows, cols, segs, s);
}

hipError_t launch_scan_step(const fdc_scan_args &a, hipStream_t s) {
  return by_dtype(a.dtype, [&](auto tag) {
    using T = decltype(tag);
    return by_lanes(a.N, [&](auto lanes) {
      constexpr int LN = decltype(lanes)::value;
      const unsigned x = (unsigned)ceil_div(a.D, 256 / LN);
      // four sequences a thread where that leaves every SIMD two waves
      if ((long long)x * a.B >= 2 * kSimds)
        return timed_launch("scan_step", k_scan_step<T, LN, 4>, dim3(x, (unsigned)ceil_div(a.B, 4)), dim3(256), 0, s, a,
                            a.D / a.G);
      return timed_launch("scan_step", k_scan_step<T, LN, 1>, dim3(x, (unsigned)a.B), dim3(256), 0, s, a, a.D / a.G);
    });
  });
}

}  // namespace fdc
