// Verification of drafted tokens (Stage 1 with a drafter; Sec. 4.1).  Included
// by opd_cache_kernels.hip only, whose double-precision exponential, scans and
// draw by inversion it uses.
//
// Sequence b has n drafted tokens x_0 .. x_{n-1}, target rows p_0 .. p_n and
// (unless the drafter is certain of its tokens: q one at them) draft rows q_0 ..
// q_{n-1}.  Token x_i is kept while u_i q_i(x_i) < p_i(x_i).  At the first that is
// not, one token is drawn from max(p_i - q_i, 0) over its sum; if all are kept,
// from p_n.  So the tokens that come out follow the target, and their log-probs
// under it are the cache's behav_logp.  All in double precision: the decisions
// and the draw are those of exact arithmetic unless a uniform lies within about
// 1e-13 of a border.
#pragma once

namespace opd {
namespace {

constexpr int kVerThreads = 256;

// A sequence's test of drafted token i.
enum Test : int { kKept = 0, kRefused = 1, kBad = 2 };

// log-sum-exps of the target rows (VerifyArgs::ws), then of the draft rows; NaN
// for a row without a distribution.
__device__ __forceinline__ double* target_lse(const VerifyArgs& a, int64_t b) {
  return a.ws + b * (a.D + 1);
}
__device__ __forceinline__ double* draft_lse(const VerifyArgs& a, int64_t b) {
  return a.ws + a.B * (a.D + 1) + b * a.D;
}

// The test of token i (any lane may make any test), from the rows' log-sum-exps.
template <class TI>
__device__ __forceinline__ int test_token(const VerifyArgs& a, int64_t b, int i) {
  const int32_t x = a.ids[b * a.D + i];
  const double L = target_lse(a, b)[i];
  const float u = a.u[b * (a.D + 1) + i];
  if ((uint32_t)x >= (uint64_t)a.V || !(L == L) || !(u >= 0.f && u < 1.f)) return kBad;
  const double p =
      exp((double)load_elem<TI>((const char*)a.target + (b * (a.D + 1) + i) * a.ld * TI::BYTES, x) - L);
  double q = 1.0;
  if (a.draft) {
    const double Lq = draft_lse(a, b)[i];
    if (!(Lq == Lq)) return kBad;
    q = exp((double)load_elem<TI>((const char*)a.draft + (b * a.D + i) * a.ldd * TI::BYTES, x) - Lq);
  }
  return (double)u * q < p ? kKept : kRefused;
}

// How many of a sequence's first `upto` tokens are kept before the first that is
// not (wave-uniform; every lane of the wave takes part).
template <class TI>
__device__ __forceinline__ int kept_tokens(const VerifyArgs& a, int64_t b, int upto, int& test) {
  const int lane = threadIdx.x & 63;
  test = kKept;
  for (int i0 = 0; i0 < upto; i0 += 64) {
    const int i = i0 + lane;
    const int t = i < upto ? test_token<TI>(a, b, i) : kKept;
    const int f = first_lane(__ballot(t != kKept));
    if (f >= 0) {
      test = __builtin_amdgcn_readlane(t, f);
      return i0 + f;
    }
  }
  return upto;
}

__device__ __forceinline__ int drafted(const VerifyArgs& a, int64_t b) {
  return a.lens ? a.lens[b] : a.D;
}

// The log-sum-exp of each target and draft row of positions [pos0, pos1) of the
// sequences whose tokens before pos0 are all kept: a workgroup per row, target
// rows first.
// (WIDE: rows of 2 GiB and more, whose offsets pass a buffer's 32 bits.)
template <class TI, bool WIDE>
__global__ void __launch_bounds__(kVerThreads) k_verify_rows(VerifyArgs a, int pos0, int pos1) {
  constexpr int W = kVerThreads / 64;
  __shared__ double tab[kExpTab];
  __shared__ float redm[W];
  __shared__ double reds[W];
  const int np = pos1 - pos0;
  const int64_t per = a.B * np;
  const bool is_draft = blockIdx.x >= per;
  const int64_t k = blockIdx.x - (is_draft ? per : 0);
  const int64_t b = k / np;
  const int i = pos0 + (int)(k - b * np);
  if (a.mask && a.mask[b] == 0) return;
  const int n = drafted(a, b);
  if (n < 0 || n > a.D || i > n || (is_draft && i >= n)) return;
  int test;
  if (pos0 > 0 && kept_tokens<TI>(a, b, pos0, test) < pos0) return;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  for (int j = tid; j < kExpTab; j += kVerThreads) tab[j] = exp2((double)j / kExpTab);
  __syncthreads();
  const char* row = is_draft ? (const char*)a.draft + (b * a.D + i) * a.ldd * TI::BYTES
                             : (const char*)a.target + (b * (a.D + 1) + i) * a.ld * TI::BYTES;
  const uint32_t nvec = (uint32_t)a.nvec;
  const uint32_t steps = (nvec + kSmpStepVecs - 1) / kSmpStepVecs;
  // one DPP row per chunk of 128 vectors; a lane of it merges its chunks
  float m = kNegInf;
  double s = 0.0;
  for (uint32_t q0 = 4u * w; q0 < steps; q0 += 4u * W) {
    float mq;
    double sq;
    chunk_record<TI, WIDE>(row, q0 + ((uint32_t)lane >> 4), q0, kSmpStepVecs, nvec, a.tail, tab, mq,
                           sq);
    const float mn = max_nan(m, mq);
    s = mn == kNegInf ? 0.0
                      : (m == kNegInf ? 0.0 : s * exp_neg((double)m - (double)mn, tab)) +
                            (mq == kNegInf ? 0.0 : sq * exp_neg((double)mq - (double)mn, tab));
    m = mn;
  }
  // the four DPP rows of each wave, then the waves
  float wm = m;
  wm = max_nan(wm, __shfl_xor(wm, 16, 64));
  wm = max_nan(wm, __shfl_xor(wm, 32, 64));
  if (lane == 0) redm[w] = wm;
  __syncthreads();
  float M = redm[0];
  for (int k2 = 1; k2 < W; ++k2) M = max_nan(M, redm[k2]);
  double sw = m == kNegInf ? 0.0 : s * exp_neg((double)m - (double)M, tab);
  sw += __shfl_xor(sw, 16, 64);
  sw += __shfl_xor(sw, 32, 64);
  if (lane == 0) reds[w] = sw;
  __syncthreads();
  if (tid == 0) {
    double S = 0.0;
    for (int k2 = 0; k2 < W; ++k2) S += reds[k2];
    const bool defined = S > 0.0 && M < __builtin_huge_valf();
    double* to = is_draft ? draft_lse(a, b) + i : target_lse(a, b) + i;
    *to = defined ? (double)M + log(S) : __builtin_nan("");
  }
}

// The masses that the last token of a sequence is drawn from.
enum Mass : int { kTarget, kResidual, kWithout };  // p; max(p - q, 0); p but for x

template <class TI>
struct DrawRow {
  const char* z;
  const char* y;  // kResidual
  double L, Lq;
  int64_t x;      // kWithout: the refused token
  int mass;
  const double* tab;
};

// This lane's eight masses of the 128-vector step at vector v0 (0 at or past c1).
template <class TI>
__device__ __forceinline__ void step_masses(const DrawRow<TI>& d, uint32_t v0, uint32_t c1,
                                            uint32_t nvec, int tail, double c2, double (&w)[8]) {
  typename TI::Vec xz[2], xy[2];
  step_load<TI>(d.z, v0, c1, nvec, tail, xz);
  if (d.mass == kResidual) step_load<TI>(d.y, v0, c1, nvec, tail, xy);
  const uint32_t v = v0 + 2u * (uint32_t)(threadIdx.x & 63);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float fz[4], fy[4];
    unpack<TI>(xz[h], fz);
    if (d.mass == kResidual) unpack<TI>(xy[h], fy);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      double p = exp_reduced((double)fz[e] - d.L, d.tab, c2);
      if (d.mass == kResidual) p = fmax(p - exp_reduced((double)fy[e] - d.Lq, d.tab, c2), 0.0);
      if (d.mass == kWithout && (int64_t)(v + h) * 4 + e == d.x) p = 0.0;
      w[4 * h + e] = v + h < c1 ? p : 0.0;
    }
  }
}

// The index drawn from the masses of chunk q: the first at which they exceed r,
// or (where rounding leaves none) the first or last of positive mass.
template <class TI>
__device__ __forceinline__ int64_t mass_element(const DrawRow<TI>& d, DrawAt at, uint32_t CV,
                                                uint32_t nvec, int tail, double c2) {
  if (at.q < 0) return -1;
  const uint32_t c0 = (uint32_t)at.q * CV, c1 = min(c0 + CV, nvec);
  double w[8];
  if (at.pick == kCross) {
    double acc = 0.0;
    for (uint32_t v0 = c0; v0 < c1; v0 += kSmpStepVecs) {
      step_masses<TI>(d, v0, c1, nvec, tail, c2, w);
      const int k = step_crossing(w, at.r, 1.0, acc);
      if (k >= 0) return (int64_t)v0 * 4 + k;
      if (k == -2) break;
    }
    at.pick = kLast;
  }
  const bool last = at.pick == kLast;
  const uint32_t nsteps = (c1 - c0 + kSmpStepVecs - 1) / kSmpStepVecs;
  for (uint32_t k = 0; k < nsteps; ++k) {
    const uint32_t v0 = c0 + (last ? nsteps - 1 - k : k) * kSmpStepVecs;
    step_masses<TI>(d, v0, c1, nvec, tail, c2, w);
    int ef = -1, eb = -1;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (w[e] > 0.0) {
        if (ef < 0) ef = e;
        eb = e;
      }
    const int vl = last ? last_lane(__ballot(eb >= 0)) : first_lane(__ballot(ef >= 0));
    if (vl >= 0) return ((int64_t)v0 + 2 * vl) * 4 + __builtin_amdgcn_readlane(last ? eb : ef, vl);
  }
  return -1;
}

struct DrawLds {
  double s[kSmpMaxChunks];  // chunk masses
  double p[kVerThreads];    // inclusive prefix of the runs
  double tab[kExpTab];
  double wt[kVerThreads / 64];
};

// A sequence's tokens: the kept ones, then the draw.  A workgroup per sequence.
template <class TI>
__global__ void __launch_bounds__(kVerThreads) k_verify_draw(VerifyArgs a) {
  constexpr int T = kVerThreads, W = T / 64;
  __shared__ DrawLds c;
  const int64_t b = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  int32_t* ids = a.ids_out + b * (a.D + 1);
  float* logp = a.logp ? a.logp + b * (a.D + 1) : nullptr;
  const int n = drafted(a, b);
  const bool masked = a.mask && a.mask[b] == 0;
  int kept = 0, test = kKept;
  if (!masked) {
    test = kBad;
    if (n >= 0 && n <= a.D) kept = kept_tokens<TI>(a, b, n, test);
  }
  for (int i = tid; i <= a.D; i += T) {
    const bool mine = !masked && i < kept;
    const int32_t x = mine ? a.ids[b * a.D + i] : -1;
    ids[i] = x;
    if (logp)
      logp[i] = mine ? (float)((double)load_elem<TI>(
                                   (const char*)a.target + (b * (a.D + 1) + i) * a.ld * TI::BYTES, x) -
                               target_lse(a, b)[i])
                     : 0.f;
  }
  if (tid == 0) a.accepted[b] = kept;
  if (masked) return;
  __syncthreads();  // (the slot of the draw is written again below)
  const float u = a.u[b * (a.D + 1) + a.D];
  DrawRow<TI> d;
  d.z = (const char*)a.target + (b * (a.D + 1) + kept) * a.ld * TI::BYTES;
  d.L = test == kBad ? __builtin_nan("") : target_lse(a, b)[kept];
  d.y = nullptr;
  d.Lq = 0.0;
  d.x = -1;
  d.mass = kTarget;
  if (test == kRefused) {
    d.mass = a.draft ? kResidual : kWithout;
    d.x = a.ids[b * a.D + kept];
    if (a.draft) {
      d.y = (const char*)a.draft + (b * a.D + kept) * a.ldd * TI::BYTES;
      d.Lq = draft_lse(a, b)[kept];
    }
  }
  if (!(d.L == d.L) || !(u >= 0.f && u < 1.f)) {
    if (tid == 0 && logp) logp[kept] = __builtin_nanf("");
    return;
  }
  for (int j = tid; j < kExpTab; j += T) c.tab[j] = exp2((double)j / kExpTab);
  __syncthreads();
  d.tab = c.tab;
  const double c2 = c2_reg();
  const uint32_t nvec = (uint32_t)a.nvec;
  const uint32_t steps = (nvec + kSmpStepVecs - 1) / kSmpStepVecs;
  const uint32_t G = (steps + kSmpMaxChunks - 1) / kSmpMaxChunks;
  const uint32_t CV = G * kSmpStepVecs, nchunk = (nvec + CV - 1) / CV;
  double S = 0.0;
  for (;;) {
    for (uint32_t q = w; q < nchunk; q += W) {
      const uint32_t c0 = q * CV, c1 = min(c0 + CV, nvec);
      double sum = 0.0;
      for (uint32_t v0 = c0; v0 < c1; v0 += kSmpStepVecs) {
        double m[8];
        step_masses<TI>(d, v0, c1, nvec, a.tail, c2, m);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += m[e];
      }
      const double all = wave_incl_scan_f64(sum);
      if (lane == 63) c.s[q] = all;
    }
    __syncthreads();
    const uint32_t C = (nchunk + T - 1) / T;
    const uint32_t r0 = min((uint32_t)tid * C, nchunk), r1 = min(r0 + C, nchunk);
    double run = 0.0;
    for (uint32_t q = r0; q < r1; ++q) run += c.s[q];
    const double incl = wave_incl_scan_f64(run);
    if (lane == 63) c.wt[w] = incl;
    __syncthreads();
    double before = 0.0;
    for (int k = 0; k < w; ++k) before += c.wt[k];
    c.p[tid] = before + incl;
    S = 0.0;
#pragma unroll
    for (int k = 0; k < W; ++k) S += c.wt[k];
    __syncthreads();
    // p(x) < q(x) leaves a residual; where rounding hides it the draw is from p
    if (S > 0.0 || d.mass == kTarget) break;
    d.mass = kTarget;
  }
  if (w != 0) return;
  const uint32_t C = (nchunk + T - 1) / T;
  const DrawAt at = smp_locate<T>(c, nchunk, C, (double)u * S, S);
  const int64_t id = mass_element<TI>(d, at, CV, nvec, a.tail, c2);
  if (lane == 0) {
    ids[kept] = (int32_t)id;
    if (logp)
      logp[kept] = id >= 0 ? (float)((double)load_elem<TI>(d.z, id) - d.L) : __builtin_nanf("");
  }
}

template <class TI>
hipError_t launch_verify_t(const VerifyArgs& a, hipStream_t stream) {
  const int64_t rows = a.B * (a.D + 1) + (a.draft ? a.B * (a.D + 1) : 0);
  if (a.nvec * (int64_t)sizeof(typename TI::Vec) < (int64_t)1 << 31)
    hipLaunchKernelGGL((k_verify_rows<TI, false>), dim3((unsigned)rows), dim3(kVerThreads), 0,
                       stream, a, 0, a.D + 1);
  else
    hipLaunchKernelGGL((k_verify_rows<TI, true>), dim3((unsigned)rows), dim3(kVerThreads), 0,
                       stream, a, 0, a.D + 1);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_verify_draw<TI>), dim3((unsigned)a.B), dim3(kVerThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_verify(const VerifyArgs& a, int in_dt, hipStream_t stream) {
  return in_dt == BF16 ? launch_verify_t<InBf16>(a, stream) : launch_verify_t<InF32>(a, stream);
}

}  // namespace opd
