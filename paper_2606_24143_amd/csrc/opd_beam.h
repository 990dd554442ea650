// Beam search beside the draws (included by opd_cache_kernels.hip only, whose sort
// keys it uses): of W beams' rows of logits, the k best
// continuations of a group, and the beams' states in their new order.
//   select   score(w, v) = scores[w] + (z[w, v] - log sum_j exp(z[w, j])),
//            the k largest of the group, ties to the lower beam, then the lower
//            token; a finished beam is a candidate as it stands
//   reorder  state[j] = state[parent[j]], in place or to another buffer
// Scores are compared in double precision, so beams that are nearly as good keep their
// order: terms of the sums of exponentials are fp32, each good to some 2e-7 (the sum of
// many different ones to about 1e-8), and doubles from a lane's vector on.
#pragma once

#include "opd_device.h"
#include "opd_model.h"

namespace opd {
namespace {

constexpr int kBeamThreads = 256;
constexpr int kBeamWaves = kBeamThreads / 64;

// The value of the lane that is S away (by exclusive or): moves within a row of 16 lanes,
// and exchanges of rows and halves, which need no LDS.
template <int S>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
  auto dpp = [](uint32_t x, auto ctrl) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xF, 0xF, true);
  };
  constexpr std::integral_constant<int, 0xB1> swap1;     // lanes 1 0 3 2 of each four
  constexpr std::integral_constant<int, 0x4E> swap2;     // 2 3 0 1
  constexpr std::integral_constant<int, 0x1B> reverse4;  // 3 2 1 0
  constexpr std::integral_constant<int, 0x141> reverse8;
  constexpr std::integral_constant<int, 0x140> reverse16;
  if constexpr (S == 1) return dpp(v, swap1);
  if constexpr (S == 2) return dpp(v, swap2);
  if constexpr (S == 4) return dpp(dpp(v, reverse8), reverse4);
  if constexpr (S == 8) return dpp(dpp(v, reverse16), reverse8);
  if constexpr (S == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return threadIdx.x & 16 ? r[0] : r[1];
  }
  if constexpr (S == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return threadIdx.x & 32 ? r[0] : r[1];
  }
}
// Lanes of `in` below this one.
__device__ __forceinline__ uint32_t lanes_below(uint64_t in) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(in >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)in, 0));
}
template <int S = 32>
__device__ __forceinline__ float lanes_max(float v) {
  v = fmaxf(v, __uint_as_float(lane_xor<S>(__float_as_uint(v))));
  if constexpr (S > 1) v = lanes_max<S / 2>(v);
  return v;
}
template <int S = 32>
__device__ __forceinline__ double lanes_sum(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint64_t o = (uint64_t)lane_xor<S>((uint32_t)(b >> 32)) << 32 | lane_xor<S>((uint32_t)b);
  v += __builtin_bit_cast(double, o);
  if constexpr (S > 1) v = lanes_sum<S / 2>(v);
  return v;
}
// A bound that k lanes' keys at least are not below: the k-th largest key, without its bits
// below LOW.  Two bits at a time, as each waits for the count of the one before.
template <int LOW>
__device__ __forceinline__ uint32_t wave_kth(uint32_t key, int k) {
  uint32_t bound = 0;
#pragma unroll
  for (int bit = 30; bit >= LOW; bit -= 2) {
    uint32_t c[3];
    bool reach[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      c[i] = bound | (uint32_t)(i + 1) << bit;
      reach[i] = __popcll(__ballot(key >= c[i])) >= k;
    }
    bound = reach[2] ? c[2] : reach[1] ? c[1] : reach[0] ? c[0] : bound;
  }
  return bound;
}
// One step of a bitonic network: lanes keep the larger where `size` and S say so.
template <int SIZE, int S>
__device__ __forceinline__ uint32_t bitonic_step(uint32_t v) {
  const int lane = threadIdx.x & 63;
  const uint32_t o = lane_xor<S>(v);
  const bool larger = ((lane & SIZE) == 0) == ((lane & S) == 0);
  return larger ? max(v, o) : min(v, o);
}
template <int SIZE, int S>
__device__ __forceinline__ uint32_t bitonic_merge(uint32_t v) {
  v = bitonic_step<SIZE, S>(v);
  if constexpr (S > 1) v = bitonic_merge<SIZE, S / 2>(v);
  return v;
}
// A value of each lane, sorted, descending.
template <int SIZE = 2>
__device__ __forceinline__ uint32_t lanes_sorted(uint32_t v) {
  v = bitonic_merge<SIZE, SIZE / 2>(v);
  if constexpr (SIZE < 64) v = lanes_sorted<SIZE * 2>(v);
  return v;
}
// The 64 largest of two descending lists, descending.
__device__ __forceinline__ uint32_t beam_merge_desc(uint32_t a, uint32_t b_reversed) {
  return bitonic_merge<64, 32>(max(a, b_reversed));
}

// Terms of a row's sum, as powers of two: f log2 e less a whole number c near its largest,
// in two multiply-adds, each exact but for the rounding of a result that is small where
// the term is large (2^-23 of it, in 1 / log2 e; the instruction's own 2^-23 is as much).
constexpr float kLog2eLow = 1.92596299e-8f;  // log2 e less its fp32 value
__device__ __forceinline__ float beam_term(float f, float c) {
  return fast_exp2(fmaf(f, kLog2eLow, fmaf(f, kLog2e, -c)));
}
// Largest magnitude of a maximum for which that holds; farther ones are subtracted first.
constexpr float kBeamNear = 65536.f;

// Candidates of a part in LDS, at most: by the bound of all lanes, all elements of fewer
// than k lanes (those above it), and a wavefront's equal to it besides.  The bound of one
// wave leaves more, as a rule fewer than four times as many.
template <class TI, int S>
constexpr uint32_t beam_cap(int k) {
  return (uint32_t)((k - 1) * S * (16 / TI::BYTES) + 64 * (16 / TI::BYTES) + k);
}

constexpr uint32_t kBeamVectors = 256;  // of a part that hold candidates
struct BeamLds {
  u32x4 vector[kBeamVectors];
  uint32_t first[kBeamVectors];  // token of each
  uint32_t top[kBeamWaves][64];
  float max[kBeamWaves];
  double sum[kBeamWaves];
  uint32_t n, vectors;
};

// One workgroup to a row's part of 256 * E * S elements, which stays in registers: its
// maximum, its sum of exponentials, and its candidates: what is not below a bound that k
// lanes' maxima reach, so k of them at least are among the best k, and none else can be.
// Bound by the vector unit (some 11 instructions an element, the exponential four times as
// long as the others).  64 groups of 8 beams, an eighth of them ended, V = 151,936 bf16:
// 30.4 us, where reading takes 20.  With elements compared out of the lanes' registers, and
// a sum for far values beside the other one (copies of all registers), 35; with the lanes'
// maxima sorted for the bound besides, 43; half as many vectors to a lane, 33.
template <class TI, int S>
__global__ void __launch_bounds__(kBeamThreads, 6) k_beam_rows(BeamArgs a) {
  constexpr int E = 16 / TI::BYTES;
  constexpr uint32_t kSpan = kBeamThreads * E;  // elements of a slot
  __shared__ BeamLds sh;
  extern __shared__ uint64_t beam_cand[];  // beam_cap
  uint64_t* const cand = beam_cand;
  const uint32_t cap = beam_cap<TI, S>(a.k);
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t row = a.row0 + blockIdx.x / a.parts;
  const uint32_t part = blockIdx.x % a.parts;
  const uint8_t done = a.finished ? a.finished[row] : 0;
  if (a.scores[row] == kNegInf || done) return;
  // (within a part: 32 bits)
  const int64_t part0 = (int64_t)part * (kSpan * S);
  const char* z = (const char*)a.logits + (row * a.ld + part0) * TI::BYTES;
  const uint32_t size = (uint32_t)min(a.V - part0, (int64_t)(kSpan * S));
  const uint32_t v0 = tid * E;
  if (tid == 0) sh.n = sh.vectors = 0;
  // (past the row's end: its last vector again, cut below)
  const uint32_t last = (size - 1) / E * E;
  u32x4 x[S];
#pragma unroll
  for (int s = 0; s < S; ++s)
    x[s] = __builtin_nontemporal_load((const u32x4*)(z + min(v0 + s * kSpan, last) * TI::BYTES));
  if (size < kSpan * S) {
#pragma unroll
    for (int s = 0; s < S; ++s) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const bool out = v0 + s * kSpan + e >= size;
        if constexpr (TI::BYTES == 2) {
          const uint32_t none = e & 1 ? 0xFF800000u : 0x0000FF80u;
          const uint32_t keep = e & 1 ? 0x0000FFFFu : 0xFFFF0000u;
          x[s][e / 2] = out ? (x[s][e / 2] & keep) | none : x[s][e / 2];
        } else {
          x[s][e] = out ? 0xFF800000u : x[s][e];
        }
      }
    }
  }
  auto value = [&](int s, int e) -> float {
    if constexpr (TI::BYTES == 2)
      return __uint_as_float(e & 1 ? x[s][e / 2] & 0xFFFF0000u : x[s][e / 2] << 16);
    else
      return __uint_as_float(x[s][e]);
  };
  // a slot's values once more, for what is rare (registers can't be indexed)
  auto slot_values = [&](int s, float (&f)[E]) {
    const uint32_t v = v0 + s * kSpan;
    const u32x4 y = *(const u32x4*)(z + min(v, last) * TI::BYTES);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if constexpr (TI::BYTES == 2)
        f[e] = __uint_as_float(e & 1 ? y[e / 2] & 0xFFFF0000u : y[e / 2] << 16);
      else
        f[e] = __uint_as_float(y[e]);
      f[e] = v + e < size ? f[e] : kNegInf;
    }
  };
  // (a NaN is a lane's maximum here, which saves quieting every operand; what the row is then
  // shows in the sum)
  float top[S], mine = kNegInf;
#pragma unroll
  for (int s = 0; s < S; ++s) {
    top[s] = value(s, 0);
#pragma unroll
    for (int e = 1; e < E; ++e) top[s] = __builtin_elementwise_maximum(top[s], value(s, e));
    mine = __builtin_elementwise_maximum(mine, top[s]);
  }
#pragma unroll
  for (int s = 0; s < S; ++s) keep_packed(x[s]);
  // What bounds the candidates from below: k lanes' maxima are not below it.  Up to 16, the
  // largest of the waves' k-th, found by the bits of the keys; more, the k-th of all.
  const uint32_t key = order_key(__float_as_uint(mine));
  uint32_t bound = 0;
  auto kth_of_all = [&]() {
    sh.top[w][lane] = lanes_sorted(key);
    __syncthreads();
    const uint32_t ab = beam_merge_desc(sh.top[0][lane], sh.top[1][63 - lane]);
    const uint32_t cd = beam_merge_desc(sh.top[2][lane], sh.top[3][63 - lane]);
    const uint32_t all = beam_merge_desc(ab, (uint32_t)__shfl((int)cd, 63 - lane, 64));
    return (uint32_t)__builtin_amdgcn_readlane((int)all, a.k - 1);
  };
  // (no key of a number is below that of the lowest; -inf has no mass)
  auto number = [](uint32_t bound) {
    return bound <= order_key(0xFF7FFFFFu) ? -3.4028234663852886e38f : key_value(bound);
  };
  if (a.k <= 16) {
    bound = wave_kth<TI::BYTES == 2 ? 16 : 8>(key, a.k);  // (bf16: keys vary above)
    const float m = lanes_max(mine);
    if (lane == 0) {
      sh.top[w][0] = bound;
      sh.max[w] = m;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kBeamWaves; ++i) bound = max(bound, sh.top[i][0]);
  } else {
    const float m = lanes_max(mine);
    if (lane == 0) sh.max[w] = m;
    bound = kth_of_all();
  }
  float m = sh.max[0];
#pragma unroll
  for (int i = 1; i < kBeamWaves; ++i) m = fmaxf(m, sh.max[i]);
  float least = number(bound);
  // Vectors with a candidate, some of a part's, to LDS: looked at element by element below
  // by all lanes, a lane's registers would each take a comparison of the wave's.
  uint64_t hit[S];
  uint32_t hits = 0, to = 0;
#pragma unroll
  for (int s = 0; s < S; ++s) {
    hit[s] = __ballot(top[s] >= least);
    hits += (uint32_t)__popcll(hit[s]);
  }
  if (lane == 0 && hits) to = atomicAdd(&sh.vectors, hits);
  to = __builtin_amdgcn_readfirstlane(to);
#pragma unroll
  for (int s = 0; s < S; ++s) {
    if (hit[s] == 0) continue;
    if (hit[s] >> lane & 1) {
      const uint32_t p = to + lanes_below(hit[s]);
      if (p < kBeamVectors) {
        sh.vector[p] = x[s];
        sh.first[p] = (uint32_t)part0 + v0 + s * kSpan;
      }
    }
    to += (uint32_t)__popcll(hit[s]);
  }

  const float off = m == kNegInf ? 0.f : m;
  const bool far = !(fabsf(off) < kBeamNear);
  const float c = far ? 0.f : rintf(off * kLog2e);
  double sum = 0.0;
  auto add = [&](const float (&t)[E]) {
    if constexpr (E == 8)
      sum += (double)(((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7])));
    else
      sum += (double)((t[0] + t[1]) + (t[2] + t[3]));
  };
  if (!far) {
#pragma unroll
    for (int s = 0; s < S; ++s) {
      float t[E];
#pragma unroll
      for (int e = 0; e < E; ++e) t[e] = beam_term(value(s, e), c);
      add(t);
    }
  } else {  // (rolled: unrolled beside the other, it costs that one copies of the registers)
#pragma unroll 1
    for (int s = 0; s < S; ++s) {
      float t[E];
      slot_values(s, t);
#pragma unroll
      for (int e = 0; e < E; ++e) t[e] = beam_term(t[e] - off, 0.f);
      add(t);
    }
  }
  sum = lanes_sum(sum);
  if (lane == 0) sh.sum[w] = sum;
  __syncthreads();
  const uint32_t vectors = sh.vectors;
  for (uint32_t i = tid; i < min(vectors, kBeamVectors) * E; i += kBeamThreads) {
    uint32_t b;
    if constexpr (TI::BYTES == 2)
      b = (uint32_t)((const uint16_t*)sh.vector)[i] << 16;
    else
      b = ((const uint32_t*)sh.vector)[i];
    if (__uint_as_float(b) >= least) {
      const uint32_t at = atomicAdd(&sh.n, 1u);
      if (at < cap) cand[at] = (uint64_t)order_key(b) << 32 | (uint32_t)~(sh.first[i / E] + i % E);
    }
  }
  __syncthreads();
  uint32_t n = sh.n;
  if (n > cap || vectors > kBeamVectors) {
    // Too many: by the bound of all lanes, those above it (in fewer than k lanes), then the
    // equal ones slot by slot, whose tokens ascend, until there are enough.
    __syncthreads();
    if (tid == 0) sh.n = 0;
    least = number(kth_of_all());
    __syncthreads();
    for (int equal = 0; equal < 2; ++equal) {
#pragma unroll 1
      for (int s = 0; s < S; ++s) {
        float f[E];
        slot_values(s, f);
        // (lanes in turn waves: a slot's tokens ascend with the lanes)
#pragma unroll 1
        for (int turn = 0; turn < kBeamWaves; ++turn) {
          const uint32_t have = sh.n;
          __syncthreads();
          if (turn == w && (!equal || have < (uint32_t)a.k)) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
              if (equal ? f[e] == least : f[e] > least) {
                const uint32_t at = atomicAdd(&sh.n, 1u);
                const uint32_t v = (uint32_t)part0 + v0 + s * kSpan + e;
                if (at < cap) cand[at] = (uint64_t)order_key(__float_as_uint(f[e])) << 32 | (uint32_t)~v;
              }
            }
          }
          __syncthreads();
        }
      }
    }
    n = sh.n;
  }
  BeamRec* rec = (BeamRec*)a.recs + (row * a.parts + part);
  uint64_t* out = a.cands + (row * a.parts + part) * (int64_t)kBeamMax;
  if (n > (uint32_t)kBeamMax) {
    // more than a record holds: the k largest, each at its rank
    for (uint32_t i = tid; i < n; i += kBeamThreads) {
      const uint64_t c = cand[i];
      uint32_t rank = 0;
      for (uint32_t o = 0; o < n; ++o) rank += cand[o] > c ? 1u : 0u;
      if (rank < (uint32_t)a.k) out[rank] = c;
    }
    n = a.k;
  } else if (tid < (int)n) {
    out[tid] = cand[tid];
  }
  if (tid == 0) {
    double t = sh.sum[0];
#pragma unroll
    for (int i = 1; i < kBeamWaves; ++i) t += sh.sum[i];
    // (from units of 2^c to units of exp(m))
    constexpr double log2e = 1.4426950408889634;
    if (!far) t *= exp2((double)c - (double)off * log2e);
    // (s NaN: a NaN or an infinity among the logits)
    *rec = BeamRec{t, m, n};
  }
}

// What a beam's candidates are scored with.
enum BeamKind : uint32_t { kBeamLive = 0, kBeamDone = 1, kBeamDead = 2, kBeamBad = 3 };
struct BeamRow {
  double l, score;  // log of the sum relative to the maximum; the beam's score
  float m;
  uint32_t kind;
};

constexpr int kMergeThreads = 1024;
constexpr int kMergeWaves = kMergeThreads / 64;
constexpr uint32_t kMergeCap = 4096;  // candidates in LDS
constexpr int kMergeEach = kMergeCap / kMergeThreads;
struct MergeLds {
  double score[kMergeCap];
  uint64_t at[kMergeCap];  // beam, token
  uint32_t rank[kMergeCap];
  BeamRow row[kBeamMax];
  uint32_t bound[2][kMergeWaves], first[2][kMergeWaves];
  uint32_t n, bad, total;
};

// a before b: a larger score, or an equal one at a lower beam, or token.
__device__ __forceinline__ bool beam_before(double sa, uint64_t a, double sb, uint64_t b) {
  return sa > sb || (sa == sb && a < b);
}
// A score's order in fp32 (equal for scores that are nearly so).
__device__ __forceinline__ uint32_t beam_key(double s) { return order_key(__float_as_uint((float)s)); }

// Of the n candidates in LDS, those that may be among the k best: what is not below a
// bound that k lanes' largest reach.  Up to 16, a wave's k-th largest serves, the best
// wave's (some 8 k are left); more take the k-th of all lanes, bit by bit.  Where that
// leaves more than `most` (scores that are equal in fp32), each one's rank decides.
__device__ __forceinline__ uint32_t merge_cut(MergeLds& sh, uint32_t n, int k, uint32_t most) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  double s[kMergeEach];
  uint64_t at[kMergeEach];
  uint32_t key[kMergeEach], top = 0;
#pragma unroll
  for (int i = 0; i < kMergeEach; ++i) {
    const uint32_t e = i * kMergeThreads + tid;
    key[i] = 0;
    s[i] = 0.0;
    at[i] = 0;
    if (e < n) {
      s[i] = sh.score[e];
      at[i] = sh.at[e];
      key[i] = beam_key(s[i]);
      top = max(top, key[i]);
    }
  }
  uint32_t bound = 0;
  if (k <= 16) {
    bound = wave_kth<8>(top, k);
    if (lane == 0) sh.bound[0][wave] = bound;
    if (tid == 0) sh.n = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kMergeWaves; ++w) bound = max(bound, sh.bound[0][w]);
  } else {
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t c = bound | (1u << bit);
      const uint32_t reach = (uint32_t)__popcll(__ballot(top >= c));
      if (lane == 0) sh.bound[bit & 1][wave] = reach;
      __syncthreads();
      uint32_t all = 0;
#pragma unroll
      for (int w = 0; w < kMergeWaves; ++w) all += sh.bound[bit & 1][w];
      if (all >= (uint32_t)k) bound = c;
    }
    if (tid == 0) sh.n = 0;
    __syncthreads();
  }
  uint64_t in[kMergeEach];
  auto reserve = [&]() {  // where a wave's go; sh.n becomes their number
    uint32_t mine = 0, to = 0;
#pragma unroll
    for (int i = 0; i < kMergeEach; ++i) {
      in[i] = __ballot(key[i] != 0);
      mine += (uint32_t)__popcll(in[i]);
    }
    if (lane == 0 && mine) to = atomicAdd(&sh.n, mine);
    __syncthreads();
    return (uint32_t)__builtin_amdgcn_readfirstlane(to);
  };
#pragma unroll
  for (int i = 0; i < kMergeEach; ++i) key[i] = key[i] < bound ? 0u : key[i];
  uint32_t to = reserve();
  uint32_t left = sh.n;
  if (left > most) {
#pragma unroll
    for (int i = 0; i < kMergeEach; ++i) {
      int rank = 0;
      for (uint32_t e = 0; e < n; ++e)
        rank += beam_before(sh.score[e], sh.at[e], s[i], at[i]) ? 1 : 0;
      key[i] = rank < k ? key[i] : 0u;
    }
    __syncthreads();
    if (tid == 0) sh.n = 0;
    __syncthreads();
    to = reserve();
    left = sh.n;
  }
#pragma unroll
  for (int i = 0; i < kMergeEach; ++i) {
    if (in[i] >> lane & 1) {
      const uint32_t p = to + lanes_below(in[i]);
      sh.score[p] = s[i];
      sh.at[p] = at[i];
    }
    to += (uint32_t)__popcll(in[i]);
  }
  __syncthreads();
  return left;
}

// One workgroup to a group: its rows' sums from their parts', the scores of the parts'
// candidates, of which LDS gets those that may be among the best, and the k best of
// them, each at its rank.  One workgroup's latencies: the records (2 us), the rows' logarithms,
// the scores in double precision, four barriers.  7.2 us for 128 records of 9 candidates; a
// wave to a record, whose lanes are mostly idle, took 9.1, all candidates through LDS 9.8.
__global__ void __launch_bounds__(kMergeThreads) k_beam_merge(BeamArgs a) {
  __shared__ MergeLds sh;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t b = blockIdx.x;
  const int W = a.W, k = a.k;
  if (tid == 0) {
    sh.bad = 0;
    sh.n = 0;
    sh.total = W;
  }
  __syncthreads();
  // The records of the group, a quarter of a wave to each (most hold fewer than 16
  // candidates): eight to a wave at a time, their first 32 candidates on their way beside
  // the rows' sums.
  const uint32_t recs = W * a.parts;
  const BeamRec* rec = (const BeamRec*)a.recs + b * recs;
  const uint64_t* cand = a.cands + b * recs * (int64_t)kBeamMax;
  constexpr int GROUPS = 2;
  constexpr uint32_t BATCH = GROUPS * kMergeWaves * 4;
  const int slot = lane & 15;
  auto record = [&](uint32_t p0, int i) {
    return p0 + (uint32_t)(i * kMergeWaves + wave) * 4 + (uint32_t)(lane >> 4);
  };
  uint64_t cs[GROUPS][2];
  uint32_t ns[GROUPS];
  auto fetch = [&](uint32_t p0) {
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      // (past a record's count, or a beam that has none, lies what the workspace held)
      const uint32_t p = min(record(p0, i), recs - 1);
      ns[i] = rec[p].n;
#pragma unroll
      for (int h = 0; h < 2; ++h) cs[i][h] = cand[(int64_t)p * kBeamMax + 16 * h + slot];
    }
  };
  fetch(0);
  for (int w = wave; w < W; w += kMergeWaves) {
    const int64_t row = b * W + w;
    const BeamRec* mine = rec + w * a.parts;
    // (a row of up to 64 parts is read once)
    BeamRec one = mine[min((uint32_t)lane, a.parts - 1)];
    const float score = a.scores[row];
    const uint8_t done = a.finished ? a.finished[row] : 0;
    BeamRow r;
    r.score = (double)score;
    r.l = 0.0;
    r.m = 0.f;
    r.kind = kBeamLive;
    if (!(score < __builtin_huge_valf())) {
      r.kind = kBeamBad;
    } else if (score == kNegInf) {
      r.kind = kBeamDead;
    } else if (done) {
      r.kind = kBeamDone;
    } else {
      float m = lane < (int)a.parts ? one.m : kNegInf;
      for (uint32_t p = lane + 64; p < a.parts; p += 64) m = fmaxf(m, mine[p].m);
      m = lanes_max(m);
      double s = 0.0;
      uint32_t found = 0;
      for (uint32_t p = lane; p < a.parts; p += 64) {
        if (p >= 64) one = mine[p];
        found += one.n;
        // (an empty part has sum 0, one with a NaN or an infinity NaN)
        const double d = one.m == kNegInf ? 0.0 : (double)one.m - (double)m;
        s += one.s * exp(d);
      }
      s = lanes_sum(s);
      if (found) atomicAdd(&sh.total, found);
      r.m = m;
      if (!(s < __builtin_huge_val()))
        r.kind = kBeamBad;
      else if (m == kNegInf)
        r.kind = kBeamDead;  // no finite logit
      else
        r.l = log(s);
    }
    if (lane == 0) {
      sh.row[w] = r;
      if (r.kind == kBeamBad) atomicOr(&sh.bad, 1u);
      if (r.kind == kBeamDone) {
        const uint32_t to = atomicAdd(&sh.n, 1u);
        sh.score[to] = r.score;
        sh.at[to] = (uint64_t)w << 32;
      }
    }
  }
  __syncthreads();
  float* scores = a.out_scores + b * k;
  int32_t* parents = a.parents + b * k;
  int32_t* ids = a.ids + b * k;
  if (sh.bad) {
    if (tid < k) {
      scores[tid] = __builtin_nanf("");
      parents[tid] = -1;
      ids[tid] = -1;
    }
    return;
  }
  uint32_t n = sh.n;
  auto reserve = [&](uint32_t count) {
    uint32_t to = 0;
    if (lane == 0 && count) to = atomicAdd(&sh.n, count);
    return (uint32_t)__builtin_amdgcn_readfirstlane(to);
  };
  auto put = [&](uint32_t w, uint64_t c, double score, uint64_t in, uint32_t to) {
    to += lanes_below(in);
    if (in >> lane & 1) {
      sh.score[to] = score;
      sh.at[to] = (uint64_t)w << 32 | (uint32_t)~(uint32_t)c;
    }
  };
  const bool fits = sh.total <= kMergeCap;
  // (of what may not fit: a wave's 64 at a time, 1,024 of the workgroup's)
  auto place = [&](uint32_t w, uint64_t c, double score, uint64_t in) {
    if (!fits && n > kMergeCap - kMergeThreads) n = merge_cut(sh, n, k, kMergeCap / 2);
    put(w, c, score, in, reserve((uint32_t)__popcll(in)));
    if (!fits) {
      __syncthreads();
      n = sh.n;
      __syncthreads();
    }
  };
  uint32_t bound = 0;  // of what k candidates are not below (k <= 16: cut before they pass LDS)
  for (uint32_t p0 = 0; p0 < recs; p0 += BATCH) {
    if (p0 > 0) fetch(p0);
    uint32_t w[GROUPS];
    BeamRow row[GROUPS];
    double ss[GROUPS][2];
    uint64_t in[GROUPS][2];
    auto score = [&](int i, uint64_t c) {
      return row[i].score + (((double)key_value((uint32_t)(c >> 32)) - (double)row[i].m) - row[i].l);
    };
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      const uint32_t p = record(p0, i);
      w[i] = min(p, recs - 1) / a.parts;
      row[i] = sh.row[w[i]];
      if (p >= recs || row[i].kind != kBeamLive) ns[i] = 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        in[i][h] = 0;
        ss[i][h] = 0.0;
        if (__ballot(ns[i] > 16u * h) == 0) continue;
        ss[i][h] = score(i, cs[i][h]);
        in[i][h] = __ballot(slot + 16u * h < ns[i] && ss[i][h] > -__builtin_huge_val());
      }
    }
    if (k <= 16) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) {
#pragma unroll
        for (int h = 0; h < 2; ++h) top = max(top, in[i][h] >> lane & 1 ? beam_key(ss[i][h]) : 0u);
      }
      top = wave_kth<8>(top, k);
      uint32_t* const first = sh.first[p0 / BATCH & 1];
      if (lane == 0) first[wave] = top;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kMergeWaves; ++i) bound = max(bound, first[i]);
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) {
#pragma unroll
        for (int h = 0; h < 2; ++h) in[i][h] &= __ballot(beam_key(ss[i][h]) >= bound);
      }
    }
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (!fits || in[i][h]) place(w[i], cs[i][h], ss[i][h], in[i][h]);
      }
    }
    // what a record holds past 32
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
#pragma unroll 1
      for (uint32_t h = 32; h < (uint32_t)kBeamMax; h += 16) {
        if (fits && __ballot(ns[i] > h) == 0) break;
        const uint64_t c = cand[(int64_t)min(record(p0, i), recs - 1) * kBeamMax + h + slot];
        const double s = score(i, c);
        place(w[i], c, s,
              __ballot(slot + h < ns[i] && s > -__builtin_huge_val() && beam_key(s) >= bound));
      }
    }
  }
  __syncthreads();
  n = sh.n;
  __syncthreads();
  while (n > 64) {
    const uint32_t left = merge_cut(sh, n, k, 1024);
    if (left == n) break;
    n = left;
  }
  // each one's rank: a candidate to a lane, a 16th of the others to a wave
  for (uint32_t i = tid; i < n; i += kMergeThreads) sh.rank[i] = 0;
  __syncthreads();
  for (uint32_t i0 = 0; i0 < n; i0 += 64) {
    const uint32_t i = min(i0 + lane, n - 1);
    const double s = sh.score[i];
    const uint64_t at = sh.at[i];
    uint32_t rank = 0;
#pragma unroll 4
    for (uint32_t e = wave; e < n; e += kMergeWaves)
      rank += beam_before(sh.score[e], sh.at[e], s, at) ? 1u : 0u;
    if (i0 + lane < n && rank) atomicAdd(&sh.rank[i], rank);
  }
  __syncthreads();
  for (uint32_t i = tid; i < n; i += kMergeThreads) {
    const uint32_t rank = sh.rank[i];
    if (rank >= (uint32_t)k) continue;
    const uint64_t at = sh.at[i];
    const int w = (int)(at >> 32);
    scores[rank] = (float)sh.score[i];
    parents[rank] = w;
    ids[rank] = sh.row[w].kind == kBeamDone ? -1 : (int32_t)(uint32_t)at;
  }
  for (int i = (int)n + tid; i < k; i += kMergeThreads) {
    scores[i] = kNegInf;
    parents[i] = -1;
    ids[i] = -1;
  }
}

// ---------------------------------------------------------------- reordering

constexpr int kMoveThreads = 256;
// A lane moves one unit of U bytes (at a slice's end what is left) of each of its group's
// states: it reads all of them before it writes, so the states may be moved in
// place; no other lane has that unit.  A beam that stays where it is is neither read nor
// written there.  KM: most beams.  States lie at any address: loads and stores of
// 16 bytes need no alignment here (32 states of 500,001 bf16 11.6 us, byte by byte 70.7; of
// 500,000 9.9).  Bound by HBM, at a copy's rate.
template <int U, int KM>
__global__ void __launch_bounds__(kMoveThreads) k_reorder(ReorderArgs a) {
  const int64_t span = a.span0 + blockIdx.x % a.spans;
  const int64_t bo = a.item0 + blockIdx.x / a.spans;  // group and outer slice
  const int64_t b = bo / a.outer, o = bo % a.outer;
  const int64_t c = (span * kMoveThreads + threadIdx.x) * U;
  if (c >= a.inner) return;
  const char* from = (const char*)a.states + b * a.W * a.stride + o * a.outer_stride;
  char* to = (char*)a.out + b * a.k * a.out_stride + o * a.out_outer_stride;
  const int32_t* parents = a.parents + b * a.k;
  auto move = [&](auto unit, int64_t c) {
    typedef decltype(unit) T;
    typedef T Any __attribute__((aligned(1)));
    T x[KM];
#pragma unroll
    for (int j = 0; j < KM; ++j) {
      if (j >= a.k) continue;
      const int32_t p = parents[j];
      x[j] = T{};
      if ((uint32_t)p >= (uint32_t)a.W || (a.in_place && p == j)) continue;
      x[j] = *(const Any*)(from + p * a.stride + c);
    }
#pragma unroll
    for (int j = 0; j < KM; ++j) {
      if (j >= a.k || (a.in_place && parents[j] == j)) continue;
      *(Any*)(to + j * a.out_stride + c) = x[j];
    }
  };
  typedef std::conditional_t<U == 16, u32x4, uint32_t> T;
  if (c + U <= a.inner) {
    move(T{}, c);
  } else if (!a.in_place && a.inner >= U) {  // the last U bytes, some of them twice
    move(T{}, a.inner - U);
  } else {
    const int left = (int)(a.inner - c);
    if constexpr (U == 16) {
      if (left & 8) move(u32x2{}, c);
      if (left & 4) move(uint32_t{}, c + (left & 8));
    }
    if (left & 2) move(uint16_t{}, c + (left & 12));
    if (left & 1) move(uint8_t{}, c + (left & 14));
  }
}

template <int U, int KM>
hipError_t reorder_u(ReorderArgs a, hipStream_t st) {
  // launches of fewer than 2^32 work-items: some items whole, or an item in parts
  constexpr int64_t most = ((int64_t)1 << 32) / kMoveThreads - 1;
  const int64_t spans = (a.inner + (int64_t)U * kMoveThreads - 1) / ((int64_t)U * kMoveThreads);
  const int64_t items = a.B * a.outer;
  const int64_t per = spans < most ? most / spans : 1;
  for (int64_t i = 0; i < items; i += per) {
    const int64_t n = items - i < per ? items - i : per;
    a.item0 = i;
    for (int64_t s0 = 0; s0 < spans; s0 += most) {
      a.span0 = s0;
      a.spans = (uint32_t)(spans - s0 < most ? spans - s0 : most);
      hipLaunchKernelGGL((k_reorder<U, KM>), dim3((unsigned)(n * a.spans)), dim3(kMoveThreads), 0,
                         st, a);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

template <class TI, int S>
hipError_t beam_s(BeamArgs a, hipStream_t st) {
  const int64_t rows = a.B * a.W;
  const int64_t most = (((int64_t)1 << 32) / kBeamThreads - 1) / a.parts;
  const size_t lds = beam_cap<TI, S>(a.k) * sizeof(uint64_t);
  for (int64_t r0 = 0; r0 < rows; r0 += most) {
    const int64_t n = rows - r0 < most ? rows - r0 : most;
    a.row0 = r0;
    hipLaunchKernelGGL((k_beam_rows<TI, S>), dim3((unsigned)(n * a.parts)), dim3(kBeamThreads), lds,
                       st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <class TI>
hipError_t beam_t(const BeamArgs& a, hipStream_t st) {
  return a.slots == 1   ? beam_s<TI, 1>(a, st)
         : a.slots == 2 ? beam_s<TI, 2>(a, st)
         : a.slots == 4 ? beam_s<TI, 4>(a, st)
                        : beam_s<TI, 8>(a, st);
}

}  // namespace

hipError_t launch_beam(const BeamArgs& a, int in_dt, hipStream_t st) {
  const hipError_t e = in_dt == BF16 ? beam_t<InBf16>(a, st) : beam_t<InF32>(a, st);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_beam_merge, dim3((unsigned)a.B), dim3(kMergeThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_reorder(const ReorderArgs& a, hipStream_t st) {
  if (a.k <= 4) return reorder_u<16, 4>(a, st);
  if (a.k <= 8) return reorder_u<16, 8>(a, st);
  if (a.k <= 16) return reorder_u<16, 16>(a, st);
  return reorder_u<4, kBeamMax>(a, st);  // (a lane holds a unit of each beam)
}

}  // namespace opd
