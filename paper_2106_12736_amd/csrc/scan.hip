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
// HBM would take a fifth of the time.
//
// LN adjacent lanes share a channel and hold four states each, so a wave owns 64 / LN channels and
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
  static constexpr int NP = 4 * LN;         // states, padded
  static constexpr int CW = 64 / LN;        // channels a wave
  static constexpr int CG = CW * kScanWaves;  // channels a workgroup
  static constexpr int E = kTok / LN;       // tokens of a block a lane does the channel's work for
  int q, ch, g, d, nvalid;                  // lane of the channel; channel in its group; group; channel; states here
  bool live;
  __device__ __forceinline__ ScanLane(const ScanGrid &sg, int N) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    q = lane % LN;
    g = blockIdx.x / sg.tiles;
    ch = (blockIdx.x - g * sg.tiles) * CG + wave * CW + lane / LN;
    live = ch < sg.Dg;
    d = g * sg.Dg + ch;
    nvalid = live ? max(0, min(4, N - 4 * q)) : 0;
  }
};

// Four states of a [.][N] float row, those that are there.
__device__ __forceinline__ void load4(float (&v)[4], const float *p, int nvalid) {
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = 0.f;
  if (nvalid > 0) {
    const Pack<float, 4> x = load_some<float, 4>(p, nvalid);
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = x.at(r);
  }
}
__device__ __forceinline__ void store4(float *p, const float (&v)[4], int nvalid) {
  if (nvalid > 0) store_some<float, 4>(p, v, nvalid);
}

// B and C of a block of tokens: each thread's share of the loads, and its way into LDS
// ([kTok][NP] floats each; zero for padded states and for tokens from `len` on).
template <class T, int LN, bool WithC>
struct BlockBC {
  static constexpr int NP = ScanLane<LN>::NP, Threads = 64 * kScanWaves;
  static constexpr int Per = (kTok * NP + Threads - 1) / Threads;
  T b[Per], c[Per];
  __device__ __forceinline__ void load(const T *Bb, int64_t sB, const T *Cb, int64_t sC, int t0, int len, int N) {
#pragma unroll
    for (int k = 0; k < Per; ++k) {
      const int i = threadIdx.x + k * Threads, s = i / NP, n = i % NP;
      const bool in = s < kTok && t0 + s < len && n < N;
      b[k] = in ? Bb[(int64_t)(t0 + s) * sB + n] : (T)0.f;
      if constexpr (WithC) c[k] = in ? Cb[(int64_t)(t0 + s) * sC + n] : (T)0.f;
    }
  }
  __device__ __forceinline__ void put(float *Bs, float *Cs) const {
#pragma unroll
    for (int k = 0; k < Per; ++k) {
      const int i = threadIdx.x + k * Threads;
      if (Per * Threads == kTok * NP || i < kTok * NP) {
        Bs[i] = (float)b[k];
        if constexpr (WithC) Cs[i] = (float)c[k];
      }
    }
  }
};

// One lane's values of a [L][D] tensor at its tokens of a block; zero outside the sequence.
template <class T, int LN>
struct LaneTokens {
  static constexpr int E = ScanLane<LN>::E;
  T v[E];
  __device__ __forceinline__ void load(const T *p, int64_t stride, int t0, int q, int len, bool live) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int t = t0 + i * LN + q;
      v[i] = live && t < len ? p[(int64_t)t * stride] : (T)0.f;
    }
  }
};

__device__ __forceinline__ float step_size(float raw, int use_softplus) {
  return use_softplus ? softplus(raw) : raw;
}

// Local: the chunk from a zero state, without outputs: its last state goes to
// carry [B][chunks][D][N], the sum of delta to dsum [B][chunks][D].  Otherwise the scan proper,
// from h0 (one chunk) or carry.
template <class T, int LN, bool Local>
__global__ __launch_bounds__(64 * kScanWaves) void k_scan_fwd(fdc_scan_args a, ScanGrid sg, float *__restrict__ carry,
                                                              float *__restrict__ dsum, float *__restrict__ saved) {
  using Lane = ScanLane<LN>;
  constexpr int NP = Lane::NP, E = Lane::E;
  __shared__ __align__(16) float Bs[2][kTok * NP], Cs[Local ? 1 : 2][Local ? 4 : kTok * NP];
  const Lane ln(sg, a.N);
  const int b = blockIdx.z, chunk = blockIdx.y;
  const int len = length_of(a.lengths, b, a.L);
  const int t_begin = chunk * sg.chunk, t_end = min(a.L, t_begin + sg.chunk);
  const int dc = ln.live ? ln.d : 0;  // a channel whose address exists
  const T *xp = static_cast<const T *>(a.x.p) + b * a.x.batch_stride + dc;
  const T *dtp = static_cast<const T *>(a.dt.p) + b * a.dt.batch_stride + dc;
  const T *gp = a.gate.p && !Local ? static_cast<const T *>(a.gate.p) + b * a.gate.batch_stride + dc : nullptr;
  const T *Bp = static_cast<const T *>(a.Bm.p) + b * a.Bm.batch_stride + ln.g * a.N;
  const T *Cp = static_cast<const T *>(a.Cm.p) + b * a.Cm.batch_stride + ln.g * a.N;
  T *yp = Local ? nullptr : static_cast<T *>(a.y.p) + b * a.y.batch_stride + dc;
  const float bias = a.dt_bias && ln.live ? a.dt_bias[dc] : 0.f, skip = a.skip && ln.live ? a.skip[dc] : 0.f;

  float A2[4], h[4];
  load4(A2, a.A + (int64_t)dc * a.N + 4 * ln.q, ln.nvalid);
#pragma unroll
  for (int r = 0; r < 4; ++r) A2[r] *= kLog2e;
  const int64_t state_at = ((int64_t)b * a.D + dc) * a.N + 4 * ln.q;
  const int64_t carry_at = (((int64_t)b * sg.chunks + chunk) * a.D + dc) * a.N + 4 * ln.q;
#pragma unroll
  for (int r = 0; r < 4; ++r) h[r] = 0.f;
  if constexpr (!Local) {
    if (sg.chunks > 1)
      load4(h, carry + carry_at, ln.nvalid);
    else if (a.h0)
      load4(h, a.h0 + state_at, ln.nvalid);
  }
  float dtotal = 0.f;

  BlockBC<T, LN, !Local> bc;
  LaneTokens<T, LN> tx, tdt, tg;
  auto fetch = [&](int t0) {
    bc.load(Bp, a.Bm.token_stride, Cp, a.Cm.token_stride, t0, len, a.N);
    tx.load(xp, a.x.token_stride, t0, ln.q, len, ln.live);
    tdt.load(dtp, a.dt.token_stride, t0, ln.q, len, ln.live);
    if (gp) tg.load(gp, a.gate.token_stride, t0, ln.q, len, ln.live);
  };
  fetch(t_begin);
  for (int t0 = t_begin, it = 0; t0 < t_end; t0 += kTok, it ^= 1) {
    float delta[E], u[E], x[E], gate[E], out[E];
    bc.put(Bs[it], Cs[Local ? 0 : it]);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      x[i] = (float)tx.v[i];
      gate[i] = gp ? (float)tg.v[i] : 0.f;
      delta[i] = ln.live && t0 + i * LN + ln.q < len ? step_size((float)tdt.v[i] + bias, a.softplus) : 0.f;
      u[i] = delta[i] * x[i];
      out[i] = 0.f;
      dtotal += delta[i];
    }
    __syncthreads();
    if (t0 + kTok < t_end) fetch(t0 + kTok);
    if constexpr (!Local)
      if (saved) store4(saved + (((int64_t)b * sg.blocks + t0 / kTok) * a.D + dc) * a.N + 4 * ln.q, h, ln.nvalid);
    if (t0 < len) {
      static_for<kTok>([&](auto step) {
        constexpr int S = decltype(step)::value, i = S / LN, src = S % LN;
        const float dl = lane_bcast<LN, src>(delta[i]), us = lane_bcast<LN, src>(u[i]);
        const float4 Bv = *reinterpret_cast<const float4 *>(&Bs[it][S * NP + 4 * ln.q]);
        const float Bq[4] = {Bv.x, Bv.y, Bv.z, Bv.w};
#pragma unroll
        for (int r = 0; r < 4; ++r) h[r] = fmaf(exp2_fast(dl * A2[r]), h[r], us * Bq[r]);
        if constexpr (!Local) {
          const float4 Cv = *reinterpret_cast<const float4 *>(&Cs[it][S * NP + 4 * ln.q]);
          float s = Cv.x * h[0];
          s = fmaf(Cv.y, h[1], s);
          s = fmaf(Cv.z, h[2], s);
          s = fmaf(Cv.w, h[3], s);
          s = lane_sum<LN>(s);
          out[i] = ln.q == src ? s : out[i];
        }
      });
    }
    if constexpr (!Local) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const int t = t0 + i * LN + ln.q;
        float v = fmaf(skip, x[i], out[i]);
        if (gp) v *= gate[i] * sigmoid(gate[i]);
        if (ln.live && t < t_end) yp[(int64_t)t * a.y.token_stride] = (T)(t < len ? v : 0.f);
      }
    }
  }
  if constexpr (Local) {
    store4(carry + carry_at, h, ln.nvalid);
    dtotal = lane_sum<LN>(dtotal);
    if (ln.live && ln.q == 0) dsum[((int64_t)b * sg.chunks + chunk) * a.D + ln.d] = dtotal;
  } else if (a.h_last && t_end == a.L) {
    store4(a.h_last + state_at, h, ln.nvalid);
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
  for (int k = 0; k < chunks; ++k) {
    const int64_t c = b * chunks + (reverse ? chunks - 1 - k : k);
    const float local = carry[c * DN + dn], decay = exp2_fast(A2 * dsum[c * D + d]);
    carry[c * DN + dn] = h;
    h = fmaf(decay, h, local);
  }
}

// The adjoint of a chunk from a zero one behind it: what reaches the state in front of the chunk.
template <class T, int LN>
__global__ __launch_bounds__(64 * kScanWaves) void k_scan_bwd_local(fdc_scan_args a, fdc_tokens gy, ScanGrid sg,
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
  const T *dtp = static_cast<const T *>(a.dt.p) + b * a.dt.batch_stride + dc;
  const T *gyp = static_cast<const T *>(gy.p) + b * gy.batch_stride + dc;
  const T *gp = a.gate.p ? static_cast<const T *>(a.gate.p) + b * a.gate.batch_stride + dc : nullptr;
  const T *Cp = static_cast<const T *>(a.Cm.p) + b * a.Cm.batch_stride + ln.g * a.N;
  const float bias = a.dt_bias && ln.live ? a.dt_bias[dc] : 0.f;
  float A2[4], g[4];
  load4(A2, a.A + (int64_t)dc * a.N + 4 * ln.q, ln.nvalid);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    A2[r] *= kLog2e;
    g[r] = 0.f;
  }
  float dtotal = 0.f;
  BlockBC<T, LN, false> cc;
  LaneTokens<T, LN> tdt, tgy, tg;
  auto fetch = [&](int t0) {
    cc.load(Cp, a.Cm.token_stride, nullptr, 0, t0, len, a.N);
    tdt.load(dtp, a.dt.token_stride, t0, ln.q, len, ln.live);
    tgy.load(gyp, gy.token_stride, t0, ln.q, len, ln.live);
    if (gp) tg.load(gp, a.gate.token_stride, t0, ln.q, len, ln.live);
  };
  const int t_last = t_begin + (t_end - t_begin - 1) / kTok * kTok;
  fetch(t_last);
  for (int t0 = t_last, it = 0; t0 >= t_begin; t0 -= kTok, it ^= 1) {
    float delta[E], gs[E];
    cc.put(Cs[it], nullptr);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float gate = gp ? (float)tg.v[i] : 0.f;
      delta[i] = ln.live && t0 + i * LN + ln.q < len ? step_size((float)tdt.v[i] + bias, a.softplus) : 0.f;
      gs[i] = (float)tgy.v[i];
      if (gp) gs[i] *= gate * sigmoid(gate);
      dtotal += delta[i];
    }
    __syncthreads();
    if (t0 > t_begin) fetch(t0 - kTok);
    if (t0 < len) {
      static_for<kTok>([&](auto step) {
        constexpr int S = kTok - 1 - decltype(step)::value, i = S / LN, src = S % LN;
        const float dl = lane_bcast<LN, src>(delta[i]), gss = lane_bcast<LN, src>(gs[i]);
        const float4 Cv = *reinterpret_cast<const float4 *>(&Cs[it][S * NP + 4 * ln.q]);
        const float Cq[4] = {Cv.x, Cv.y, Cv.z, Cv.w};
#pragma unroll
        for (int r = 0; r < 4; ++r) g[r] = exp2_fast(dl * A2[r]) * fmaf(Cq[r], gss, g[r]);
      });
    }
  }
  store4(carry + (((int64_t)b * sg.chunks + chunk) * a.D + dc) * a.N + 4 * ln.q, g, ln.nvalid);
  dtotal = lane_sum<LN>(dtotal);
  if (ln.live && ln.q == 0) dsum[((int64_t)b * sg.chunks + chunk) * a.D + ln.d] = dtotal;
}

// The backward proper.  A block's states are formed again from the saved one in front of it and
// kept in registers (16 tokens x 4 states and their decays), then the block is walked backwards.
// The sums of gB and gC over the channels: every fourth token the lanes put their four products of
// four tokens into LDS and add them up over the wave's channels the other way round; the waves'
// sums are added in wave order, and the workgroups' partial sums
// (partBC [2][tiles][B][L][G N]) by k_scan_sum_bc.  partP [B chunks][D N + 2 D]: gA, gskip, gdt_bias.
template <class T, int LN>
__global__ __launch_bounds__(64 * kScanWaves) void k_scan_bwd(fdc_scan_args a, fdc_scan_grads gr, ScanGrid sg,
                                                              const float *__restrict__ saved,
                                                              const float *__restrict__ carry,
                                                              float *__restrict__ partBC,
                                                              float *__restrict__ partP) {
  using Lane = ScanLane<LN>;
  constexpr int NP = Lane::NP, E = Lane::E, CW = Lane::CW;
  constexpr int kSteps = 4;                   // tokens a round of the channel sums takes
  constexpr int Row = 64 * 4 + 16;            // floats of one (token, kind): the lanes' four each, and a shift of banks
  constexpr int Outs = kSteps * 2 * LN;       // float4 sums a round forms
  constexpr int Parts = Outs < 64 ? 64 / Outs : 1;  // lanes that share one
  constexpr int Rounds = Outs < 64 ? 1 : Outs / 64;
  constexpr int Sum = CW / Parts;             // channels a lane adds
  __shared__ __align__(16) float Bs[kTok * NP], Cs[kTok * NP];
  __shared__ __align__(16) float prod[kScanWaves][kSteps * 2 * Row];
  __shared__ __align__(16) float wsum[kScanWaves][kTok * 2 * NP];
  const Lane ln(sg, a.N);
  const int b = blockIdx.z, chunk = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int len = length_of(a.lengths, b, a.L);
  const int t_begin = chunk * sg.chunk, t_end = min(a.L, t_begin + sg.chunk);
  const int dc = ln.live ? ln.d : 0;
  const T *xp = static_cast<const T *>(a.x.p) + b * a.x.batch_stride + dc;
  const T *dtp = static_cast<const T *>(a.dt.p) + b * a.dt.batch_stride + dc;
  const T *gyp = static_cast<const T *>(gr.gy.p) + b * gr.gy.batch_stride + dc;
  const T *gp = a.gate.p ? static_cast<const T *>(a.gate.p) + b * a.gate.batch_stride + dc : nullptr;
  const T *Bp = static_cast<const T *>(a.Bm.p) + b * a.Bm.batch_stride + ln.g * a.N;
  const T *Cp = static_cast<const T *>(a.Cm.p) + b * a.Cm.batch_stride + ln.g * a.N;
  T *gxp = static_cast<T *>(gr.gx.p) + b * gr.gx.batch_stride + dc;
  T *gdtp = static_cast<T *>(gr.gdt.p) + b * gr.gdt.batch_stride + dc;
  T *ggp = gp ? static_cast<T *>(gr.ggate.p) + b * gr.ggate.batch_stride + dc : nullptr;
  const float bias = a.dt_bias && ln.live ? a.dt_bias[dc] : 0.f, skip = a.skip && ln.live ? a.skip[dc] : 0.f;
  const int tile = blockIdx.x - ln.g * sg.tiles;
  const int64_t GN = (int64_t)a.G * a.N, kind_stride = (int64_t)sg.tiles * a.B * a.L * GN;
  float *pbc = partBC + ((int64_t)tile * a.B + b) * a.L * GN + ln.g * a.N;

  float A2[4], g[4], gA[4], gskip = 0.f, gbias = 0.f;
  load4(A2, a.A + (int64_t)dc * a.N + 4 * ln.q, ln.nvalid);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    A2[r] *= kLog2e;
    g[r] = gA[r] = 0.f;
  }
  if (sg.chunks > 1) load4(g, carry + (((int64_t)b * sg.chunks + chunk) * a.D + dc) * a.N + 4 * ln.q, ln.nvalid);

  BlockBC<T, LN, true> bc;
  LaneTokens<T, LN> tx, tdt, tg, tgy;
  float hs[4];
  auto fetch = [&](int t0) {
    bc.load(Bp, a.Bm.token_stride, Cp, a.Cm.token_stride, t0, len, a.N);
    tx.load(xp, a.x.token_stride, t0, ln.q, len, ln.live);
    tdt.load(dtp, a.dt.token_stride, t0, ln.q, len, ln.live);
    tgy.load(gyp, gr.gy.token_stride, t0, ln.q, len, ln.live);
    if (gp) tg.load(gp, a.gate.token_stride, t0, ln.q, len, ln.live);
    load4(hs, saved + (((int64_t)b * sg.blocks + t0 / kTok) * a.D + dc) * a.N + 4 * ln.q, ln.nvalid);
  };
  const int t_last = t_begin + (t_end - t_begin - 1) / kTok * kTok;
  fetch(t_last);
  for (int t0 = t_last; t0 >= t_begin; t0 -= kTok) {
    float delta[E], u[E], x[E], gs[E], out[E], gu[E], gd[E], gate[E], gyv[E], raw[E];
    bc.put(Bs, Cs);
    float h[kTok + 1][4], dec[kTok][4];
#pragma unroll
    for (int r = 0; r < 4; ++r) h[0][r] = hs[r];
#pragma unroll
    for (int i = 0; i < E; ++i) {
      x[i] = (float)tx.v[i];
      gate[i] = gp ? (float)tg.v[i] : 0.f;
      gyv[i] = (float)tgy.v[i];
      raw[i] = (float)tdt.v[i] + bias;
      delta[i] = ln.live && t0 + i * LN + ln.q < len ? step_size(raw[i], a.softplus) : 0.f;
      u[i] = delta[i] * x[i];
      gs[i] = gp ? gyv[i] * gate[i] * sigmoid(gate[i]) : gyv[i];
      out[i] = gu[i] = gd[i] = 0.f;
    }
    __syncthreads();
    if (t0 > t_begin) fetch(t0 - kTok);
    if (t0 < len) {
      static_for<kTok>([&](auto step) {
        constexpr int S = decltype(step)::value, i = S / LN, src = S % LN;
        const float dl = lane_bcast<LN, src>(delta[i]), us = lane_bcast<LN, src>(u[i]);
        const float4 Bv = *reinterpret_cast<const float4 *>(&Bs[S * NP + 4 * ln.q]);
        const float Bq[4] = {Bv.x, Bv.y, Bv.z, Bv.w};
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          dec[S][r] = exp2_fast(dl * A2[r]);
          h[S + 1][r] = fmaf(dec[S][r], h[S][r], us * Bq[r]);
        }
      });
      static_for<kTok / kSteps>([&](auto round) {
        constexpr int R = kTok / kSteps - 1 - decltype(round)::value;
        static_for<kSteps>([&](auto step) {
          constexpr int K = kSteps - 1 - decltype(step)::value, S = R * kSteps + K, i = S / LN, src = S % LN;
          const float dl = lane_bcast<LN, src>(delta[i]), us = lane_bcast<LN, src>(u[i]);
          const float gss = lane_bcast<LN, src>(gs[i]);
          const float4 Bv = *reinterpret_cast<const float4 *>(&Bs[S * NP + 4 * ln.q]);
          const float4 Cv = *reinterpret_cast<const float4 *>(&Cs[S * NP + 4 * ln.q]);
          const float Bq[4] = {Bv.x, Bv.y, Bv.z, Bv.w}, Cq[4] = {Cv.x, Cv.y, Cv.z, Cv.w};
          float su = 0.f, sd = 0.f, sy = 0.f, pB[4], pC[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            g[r] = fmaf(Cq[r], gss, g[r]);
            pB[r] = g[r] * us;
            pC[r] = h[S + 1][r] * gss;
            su = fmaf(g[r], Bq[r], su);
            sy = fmaf(Cq[r], h[S + 1][r], sy);
            g[r] *= dec[S][r];
            const float e = g[r] * h[S][r];
            sd = fmaf(e, A2[r], sd);
            gA[r] = fmaf(e, dl, gA[r]);
          }
          float *pw = &prod[wave][K * 2 * Row + 4 * lane];
          *reinterpret_cast<float4 *>(pw) = make_float4(pB[0], pB[1], pB[2], pB[3]);
          *reinterpret_cast<float4 *>(pw + Row) = make_float4(pC[0], pC[1], pC[2], pC[3]);
          su = lane_sum<LN>(su);
          sd = lane_sum<LN>(sd);
          sy = lane_sum<LN>(sy);
          gu[i] = ln.q == src ? su : gu[i];
          gd[i] = ln.q == src ? sd : gd[i];
          out[i] = ln.q == src ? sy : out[i];
        });
        wave_sync();
#pragma unroll
        for (int k = 0; k < Rounds; ++k) {
          // this lane's sum: (token, kind) `row`, states 4 oq .. 4 oq + 3, over `Sum` of the channels
          const int o = (lane + 64 * k) % Outs, row = o / LN, oq = o % LN, first = lane / (Outs < 64 ? Outs : 64) * Sum;
          const float *pr = &prod[wave][row * Row + 4 * (first * LN + oq)];
          float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int c = 0; c < Sum; ++c) {
            const float4 v = *reinterpret_cast<const float4 *>(pr + 4 * c * LN);
            s[0] += v.x, s[1] += v.y, s[2] += v.z, s[3] += v.w;
          }
#pragma unroll
          for (int off = Outs; off < 64; off <<= 1)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[r] += __shfl_xor(s[r], off, 64);
          if (Parts == 1 || lane < Outs)
            *reinterpret_cast<float4 *>(&wsum[wave][(R * kSteps * 2 + row) * NP + 4 * oq]) =
                make_float4(s[0], s[1], s[2], s[3]);
        }
        wave_sync();
      });
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int t = t0 + i * LN + ln.q;
      const bool in = t < len;
      gd[i] = fmaf(gd[i], kLn2, gu[i] * x[i]);
      if (a.softplus) gd[i] *= sigmoid(raw[i]);
      if (!in) gd[i] = 0.f;
      gskip = fmaf(gs[i], x[i], gskip);
      gbias += gd[i];
      if (ln.live && t < t_end) {
        gxp[(int64_t)t * gr.gx.token_stride] = (T)(in ? fmaf(gu[i], delta[i], gs[i] * skip) : 0.f);
        gdtp[(int64_t)t * gr.gdt.token_stride] = (T)gd[i];
        if (gp) {
          const float sg_ = sigmoid(gate[i]);
          const float v = gyv[i] * fmaf(skip, x[i], out[i]) * (sg_ * (1.f + gate[i] * (1.f - sg_)));
          ggp[(int64_t)t * gr.ggate.token_stride] = (T)(in ? v : 0.f);
        }
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kTok * 2 * NP; i += 64 * kScanWaves) {
      const int s = i / (2 * NP), kind = i / NP % 2, n = i % NP;
      float v = 0.f;
      if (t0 < len)
#pragma unroll
        for (int w = 0; w < kScanWaves; ++w) v += wsum[w][i];
      if (n < a.N && t0 + s < t_end) pbc[kind * kind_stride + (int64_t)(t0 + s) * GN + n] = v;
    }
  }
  float *pp = partP + ((int64_t)b * sg.chunks + chunk) * ((int64_t)a.D * a.N + 2 * a.D);
  store4(pp + (int64_t)dc * a.N + 4 * ln.q, gA, ln.nvalid);
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

// One token: LN lanes a (sequence, channel); a pass over the states (HBM: 8 bytes a state).
template <class T, int LN>
__global__ __launch_bounds__(256) void k_scan_step(fdc_scan_args a, int Dg) {
  const int i = blockIdx.x * (256 / LN) + threadIdx.x / LN, q = threadIdx.x % LN, b = blockIdx.y;
  const bool live = i < a.D;
  const int d = live ? i : 0, g = d / Dg, nvalid = live ? max(0, min(4, a.N - 4 * q)) : 0;
  const float x = (float)static_cast<const T *>(a.x.p)[b * a.x.batch_stride + d];
  const float raw = (float)static_cast<const T *>(a.dt.p)[b * a.dt.batch_stride + d] + (a.dt_bias ? a.dt_bias[d] : 0.f);
  const float gate = a.gate.p ? (float)static_cast<const T *>(a.gate.p)[b * a.gate.batch_stride + d] : 0.f;
  const int64_t at = ((int64_t)b * a.D + d) * a.N + 4 * q;
  float A[4], h[4], s = 0.f;
  load4(A, a.A + (int64_t)d * a.N + 4 * q, nvalid);
  load4(h, a.h0 + at, nvalid);
  Pack<T, 4> Bv{}, Cv{};
  if (nvalid > 0) {
    Bv = load_some<T, 4>(static_cast<const T *>(a.Bm.p) + b * a.Bm.batch_stride + g * a.N + 4 * q, nvalid);
    Cv = load_some<T, 4>(static_cast<const T *>(a.Cm.p) + b * a.Cm.batch_stride + g * a.N + 4 * q, nvalid);
  }
  const float delta = step_size(raw, a.softplus), u = delta * x;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    h[r] = fmaf(exp2_fast(delta * (A[r] * kLog2e)), h[r], u * Bv.at(r));
    s = fmaf(Cv.at(r), h[r], s);
  }
  store4(a.h_last + at, h, nvalid);
  s = lane_sum<LN>(s);
  if (a.skip) s = fmaf(a.skip[d], x, s);
  if (a.gate.p) s *= gate * sigmoid(gate);
  if (live && q == 0) static_cast<T *>(a.y.p)[b * a.y.batch_stride + d] = (T)s;
}

namespace {

int lanes_of(int N) { return N <= 8 ? 2 : N <= 16 ? 4 : N <= 32 ? 8 : 16; }

// As many chunks as bring the waves of the launch to kWantWaves where the channels alone give too few.
constexpr int kWantWaves = 2048;  // two a SIMD
ScanGrid scan_grid(int B, int L, int D, int N, int G) {
  ScanGrid sg;
  sg.Dg = D / G;
  sg.tiles = (int)ceil_div(sg.Dg, 64 / lanes_of(N) * kScanWaves);
  sg.blocks = (int)ceil_div(L, kTok);
  const long long waves = (long long)B * G * sg.tiles * kScanWaves;
  long long chunks = waves * 2 > kWantWaves ? 1 : std::min<long long>(ceil_div(kWantWaves, waves), ceil_div(sg.blocks, 4));
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
  return carry_floats(scan_grid(B, L, D, N, G), B, D, N);
}
size_t scan_bwd_ws_floats(int B, int L, int D, int N, int G) {
  const ScanGrid sg = scan_grid(B, L, D, N, G);
  return carry_floats(sg, B, D, N) + round4((size_t)B * sg.chunks * ((size_t)D * N + 2 * D)) +
         round4((size_t)2 * sg.tiles * B * L * G * N);
}

hipError_t launch_scan_fwd(const fdc_scan_args &a, float *saved, float *ws, hipStream_t s) {
  const ScanGrid sg = scan_grid(a.B, a.L, a.D, a.N, a.G);
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
  const ScanGrid sg = scan_grid(a.B, a.L, a.D, a.N, a.G);
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
      return timed_launch("scan_step", k_scan_step<T, LN>, dim3((unsigned)ceil_div(a.D, 256 / LN), (unsigned)a.B),
                          dim3(256), 0, s, a, a.D / a.G);
    });
  });
}

}  // namespace fdc
