// Verification of drafted tokens (Stage 1 with a drafter; Sec. 4.1).  Included
// by opd_cache_kernels.hip only, whose double-precision exponentials, scans and
// draw by inversion it uses.
//
// Sequence b has n drafted tokens x_0 .. x_{n-1}, target rows p_0 .. p_n and
// (unless the drafter is certain of its tokens: q one at them) draft rows q_0 ..
// q_{n-1}.  Token x_i is kept while u_i q_i(x_i) < p_i(x_i).  At the first that is
// not, one token is drawn from max(p_i - q_i, 0) over its sum; if all are kept,
// from p_n.  So the tokens that come out follow the target, and their log-probs
// under it are the cache's behav_logp.  All in double precision, relative to a
// row's maximum where its logits lie far from 0: the decisions and the draw are
// those of exact arithmetic unless u q and p differ by less than about 1e-13 of p,
// or the draw's uniform lies as near to a cumulative mass.
//
// k_verify_rows sums the rows, k_verify_draw draws.  Rows past a sequence's first
// refusal have no part in the result, and they are an eighth to three quarters of
// all rows.  So the positions are summed in rounds, a launch each (launch_verify_t): a
// round leaves out the sequences that the rounds before it ended.
#pragma once

namespace opd {
namespace {

constexpr int kVerThreads = 512;
constexpr int kVerWaves = kVerThreads / 64;
// Sums of exp(z) itself, not of exp(z - max), need no maximum: a double holds them
// for logits below 640.  A part of a row with others, or whose sum is so small that
// its terms may have been cut off, is summed again relative to its maximum.
constexpr float kVerTop = 640.f;
constexpr double kVerMinSum = 8.75651076269652e-27;  // exp(-60)

// A sequence's test of drafted token i (0: not made).
enum Test : uint32_t { kUntested = 0, kKept = 1, kRefused = 2, kBad = 3 };

// What a part of a row sums to: s exp(m) (s NaN: no distribution), m 0 as a rule.
struct VerRec {
  double m, s;
};
// A row sums to exp(m + l): m the largest of its parts', l NaN without a
// distribution.  Kept apart, since far from 0 the sum m + l is m: log p(z) is (z - m)
// - l, of a difference exact to 2^-53 of itself.
struct VerRow {
  double l, m;
};
__device__ __forceinline__ double log_p(float z, const VerRow& r) { return ((double)z - r.m) - r.l; }

// LDS of the terms: the 512 powers of the exponential, and exp(z) of each bf16 z.
template <bool TABLE>
struct VerTab {
  double p[kExpTab];
  double e[TABLE ? kTabSize + 2 : 1];
};

template <bool TABLE, int T>
__device__ __forceinline__ void ver_setup(VerTab<TABLE>& t, double* scratch) {
  for (int j = threadIdx.x; j < kExpTab; j += T) t.p[j] = exp2((double)j / kExpTab);
  if constexpr (TABLE)
    tab_setup<T>(t.e, scratch);
  else
    __syncthreads();
}

// Eight consecutive elements of a row.
template <class TI>
struct Group;
template <>
struct Group<InBf16> {
  u32x4 x;
};
template <>
struct Group<InF32> {
  u32x4 x, y;
};
// (the whole group lies in the row)
template <class TI>
__device__ __forceinline__ Group<TI> group_load(const char* row, uint32_t g) {
  Group<TI> r;
  const u32x4* p = (const u32x4*)(row + (size_t)g * 8 * TI::BYTES);
  r.x = __builtin_nontemporal_load(p);
  if constexpr (TI::BYTES == 4) r.y = __builtin_nontemporal_load(p + 1);
  return r;
}
// (elements at or past V, and groups at or past g1, read as -inf)
template <class TI>
__device__ __forceinline__ Group<TI> group_load_end(const char* row, uint32_t g, uint32_t g1,
                                                    int64_t V) {
  if (g < g1 && (int64_t)g * 8 + 8 <= V) return group_load<TI>(row, g);
  Group<TI> r;
  if constexpr (TI::BYTES == 2) {
    r.x = u32x4{0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u};
  } else {
    r.x = u32x4{0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u};
    r.y = r.x;
  }
  if (g < g1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if ((int64_t)g * 8 + e >= V) continue;
      if constexpr (TI::BYTES == 2) {
        const uint32_t b = ((const uint16_t*)row)[(size_t)g * 8 + e];
        r.x[e / 2] = e & 1 ? (r.x[e / 2] & 0xFFFFu) | b << 16 : (r.x[e / 2] & 0xFFFF0000u) | b;
      } else {
        const uint32_t b = ((const uint32_t*)row)[(size_t)g * 8 + e];
        if (e < 4)
          r.x[e & 3] = b;
        else
          r.y[e & 3] = b;
      }
    }
  }
  return r;
}
template <class TI>
__device__ __forceinline__ void group_values(const Group<TI>& g, float (&f)[8]) {
  if constexpr (TI::BYTES == 2) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      f[2 * d] = __uint_as_float(g.x[d] << 16);
      f[2 * d + 1] = __uint_as_float(g.x[d] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      f[d] = __uint_as_float(g.x[d]);
      f[4 + d] = __uint_as_float(g.y[d]);
    }
  }
}

// The table offsets of a group's logits, if the table holds a wavefront's.  Logits
// below -820 (masked actions and what lies past a row, -inf) read the entry past the
// table, which is 0, as exp_reduced gives.  A wavefront with others (zeros, [-820, -640],
// 640 and more) takes the exponential for its group.  5% of the entries of every row,
// with the table / without it, us: 64 sequences of 5 drafts, V = 151,936, ordinary 77 / 97,
// -inf 82 / 94, zeros 125 / 95; 512 of 8, ordinary 300 / 432, -inf 320 / 438, zeros 638 / 455.
__device__ __forceinline__ bool table_offsets(const u32x4& x, u16x2 (&t)[4]) {
  u16x2 top = {0, 0};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    t[k] = tab_index(x[k]);
    top = __builtin_elementwise_max(top, t[k]);
  }
  if (__ballot(top[0] >= kTabSize || top[1] >= kTabSize) == 0) return true;
  const TabRare rare;
  const u16x2 size = pair_of(kTabSize);
  top = (u16x2){0, 0};
#pragma unroll
  for (int k = 0; k < 4; ++k) top = __builtin_elementwise_max(top, rare(t[k]));
  if (__ballot(top[0] >= kTabSize || top[1] >= kTabSize) != 0) return false;
#pragma unroll
  for (int k = 0; k < 4; ++k) t[k] = __builtin_elementwise_min(t[k], size);
  return true;
}

// exp(z) of a group's elements; rare is set where one is not below kVerTop.  By
// the table, where a wavefront's values are all of magnitude [2^-17, 640) or below
// -820, one LDS read each.
template <class TI, bool TABLE>
__device__ __forceinline__ void group_terms(const Group<TI>& g, const VerTab<TABLE>& tab,
                                            double c2, bool& rare, double (&w)[8]) {
  if constexpr (TABLE) {
    u16x2 t[4];
    if (table_offsets(g.x, t)) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        w[2 * k] = tab.e[t[k][0]];
        w[2 * k + 1] = tab.e[t[k][1]];
      }
      return;
    }
  }
  float f[8];
  group_values<TI>(g, f);
  float top = f[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) top = max_nan(top, f[e]);
  rare |= !(top < kVerTop);
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = exp_reduced((double)f[e], tab.p, c2);
}

// ---------------------------------------------------------------- sums of the rows

__device__ __forceinline__ double wave_sum_f64(double v) {  // the same in every lane
  return from_lane(wave_incl_scan_f64(v), 63);
}

// The record of groups [g0, g1) of a row, by one wavefront, in tiles of K groups per
// lane.
template <class TI>
constexpr int ver_k() { return TI::BYTES == 2 ? 4 : 2; }
template <class TI, bool TABLE>
__device__ __forceinline__ VerRec part_record(const char* row, uint32_t g0, uint32_t g1, int64_t V,
                                              const VerTab<TABLE>& tab) {
  constexpr int K = ver_k<TI>();
  const uint32_t lane = threadIdx.x & 63;
  const double c2 = c2_reg();
  const uint32_t full = min(g1, (uint32_t)(V >> 3));  // groups that lie in the row
  double acc[4] = {0.0, 0.0, 0.0, 0.0};
  bool rare = false;
  auto add = [&](const Group<TI>& g) {
    if constexpr (TABLE) {
      u16x2 t[4];
      if (table_offsets(g.x, t)) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          acc[k] += tab.e[t[k][0]];
          acc[k] += tab.e[t[k][1]];
        }
      } else {  // (two exponentials at a time: eight spill)
#pragma unroll 1
        for (int k = 0; k < 4; ++k) {
          const uint32_t x = k < 2 ? (k ? g.x[1] : g.x[0]) : (k & 1 ? g.x[3] : g.x[2]);
          const float f = __uint_as_float(x << 16), h = __uint_as_float(x & 0xFFFF0000u);
          rare |= !(max_nan(f, h) < kVerTop);
          acc[0] += exp_reduced((double)f, tab.p, c2);
          acc[1] += exp_reduced((double)h, tab.p, c2);
        }
      }
    } else {
      double v[8];
      group_terms<TI, TABLE>(g, tab, c2, rare, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e & 3] += v[e];
    }
    __builtin_amdgcn_sched_barrier(0);  // (a group at a time: more do not fit the registers)
  };
  auto load = [&](Group<TI> (&x)[K], uint32_t at) {
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = group_load<TI>(row, at + 64 * k + lane);
  };
  uint32_t at = g0;
  int tiles = full > g0 ? (int)((full - g0) / (64u * K)) : 0;
  if (tiles > 0) {
    Group<TI> x[K], y[K];
    load(x, at);
    // (two tiles a turn, the next one on its way meanwhile)
    for (; tiles > 2; tiles -= 2, at += 128u * K) {
      load(y, at + 64u * K);
#pragma unroll
      for (int k = 0; k < K; ++k) add(x[k]);
      load(x, at + 128u * K);
#pragma unroll
      for (int k = 0; k < K; ++k) add(y[k]);
    }
    if (tiles == 2) load(y, at + 64u * K);
#pragma unroll
    for (int k = 0; k < K; ++k) add(x[k]);
    if (tiles == 2) {
#pragma unroll
      for (int k = 0; k < K; ++k) add(y[k]);
    }
    at += 64u * K * tiles;
  }
#pragma unroll 1
  for (; at < g1; at += 64) add(group_load_end<TI>(row, at + lane, g1, V));
  const double s = wave_sum_f64((acc[0] + acc[1]) + (acc[2] + acc[3]));
  if (__ballot(rare) == 0 && s >= kVerMinSum) return VerRec{0.0, s};
  float m = kNegInf;
#pragma unroll 1
  for (uint32_t g = g0 + lane; g < g1; g += 64) {
    float f[8];
    group_values<TI>(group_load_end<TI>(row, g, g1, V), f);
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max_nan(m, f[e]);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) m = max_nan(m, __shfl_xor(m, o, 64));
  if (m == kNegInf) return VerRec{(double)kNegInf, 0.0};
  if (!(m < __builtin_huge_valf())) return VerRec{0.0, __builtin_nan("")};
  double t = 0.0;
#pragma unroll 1
  for (uint32_t g = g0 + lane; g < g1; g += 64) {
    float f[8];
    group_values<TI>(group_load_end<TI>(row, g, g1, V), f);
#pragma unroll
    for (int e = 0; e < 8; ++e) t += term(f[e], (double)m, tab.p, c2);
  }
  return VerRec{(double)m, wave_sum_f64(t)};
}

// Words and doubles that workgroups pass each other within a launch: device-scope
// stores go through to where every XCD's device-scope loads read.  shared_wait()
// between such stores and the counter that announces them: they have arrived.  (A
// release fence would write back the XCD's whole L2 as well, which cost 130 of
// 160 us at 64 sequences.)
__device__ __forceinline__ void shared_wait() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0);
  asm volatile("" ::: "memory");
}
template <class T>
__device__ __forceinline__ T shared_load(const T* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <class T>
__device__ __forceinline__ void shared_store(T* p, T v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The workspace: rows (target, then draft), their parts, chunk masses, then the
// words that start at 0.
struct VerWs {
  VerRow* row;
  VerRec* rec;
  double* mass;
  uint32_t *test, *count, *stop, *done;
};
__device__ __forceinline__ VerWs ver_ws(const VerifyArgs& a) {
  VerWs w;
  const int64_t R = a.B * (2 * a.D + 1);
  w.row = (VerRow*)a.ws;
  w.rec = (VerRec*)(w.row + R);
  w.mass = (double*)(w.rec + R * a.parts);
  w.test = (uint32_t*)(w.mass + (a.draw_parts > 1 ? a.B * (int64_t)a.nchunk : 0));
  w.count = w.test + a.B * (a.D + 1);
  w.stop = w.count + a.B * (a.D + 1);
  w.done = w.stop + a.B;
  return w;
}
__device__ __forceinline__ int64_t target_row(const VerifyArgs& a, int64_t b, int i) {
  return b * (a.D + 1) + i;
}
__device__ __forceinline__ int64_t draft_row(const VerifyArgs& a, int64_t b, int i) {
  return b * a.D + i;
}
template <class TI>
__device__ __forceinline__ const char* target_ptr(const VerifyArgs& a, int64_t b, int i) {
  return (const char*)a.target + target_row(a, b, i) * a.ld * TI::BYTES;
}
template <class TI>
__device__ __forceinline__ const char* draft_ptr(const VerifyArgs& a, int64_t b, int i) {
  return (const char*)a.draft + draft_row(a, b, i) * a.ldd * TI::BYTES;
}
__device__ __forceinline__ int drafted(const VerifyArgs& a, int64_t b) {
  if (a.mask && a.mask[b] == 0) return -1;
  const int n = a.lens ? a.lens[b] : a.D;
  return n > a.D ? -1 : n;
}

// A row from its parts (at most 64, one to a lane; the order of the sum is fixed).
__device__ __forceinline__ VerRow row_of_parts(const VerRec* r, int parts, const double* tab) {
  const int lane = threadIdx.x & 63;
  VerRec x{(double)kNegInf, 0.0};
  if (lane < parts) x = VerRec{shared_load(&r[lane].m), shared_load(&r[lane].s)};
  double m = x.m;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) m = fmax(m, __shfl_xor(m, o, 64));
  if (m == (double)kNegInf) return VerRow{__builtin_nan(""), m};
  const double s = wave_sum_f64(x.s * (x.m == m ? 1.0 : exp_neg(x.m - m, tab)));
  return VerRow{log(s), m};
}

// The test of token i of sequence b, its rows summed (one lane).
template <class TI>
__device__ __forceinline__ uint32_t test_token(const VerifyArgs& a, int64_t b, int i,
                                               const VerRow& rt, const VerRow& rd,
                                               const double* tab) {
  const int32_t x = a.ids[b * a.D + i];
  const float u = a.u[b * (a.D + 1) + i];
  if ((uint64_t)(uint32_t)x >= (uint64_t)a.V || !(rt.l == rt.l) || !(rd.l == rd.l) ||
      !(u >= 0.f && u < 1.f))
    return kBad;
  const double p = exp_neg(log_p(load_elem<TI>(target_ptr<TI>(a, b, i), x), rt), tab);
  const double q =
      a.draft ? exp_neg(log_p(load_elem<TI>(draft_ptr<TI>(a, b, i), x), rd), tab) : 1.0;
  return (double)u * q < p ? kKept : kRefused;
}

__global__ void __launch_bounds__(256) k_verify_clear(uint32_t* words, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256)
    words[i] = 0u;
}

// The rows of positions [pos0, pos1) that the sequences still need: of sequence b,
// `targets` and then `drafts` rows from pos0 on.
struct RoundRows {
  int targets, drafts;
};
__device__ __forceinline__ RoundRows round_rows(const VerifyArgs& a, const VerWs& ws, int64_t b,
                                                int pos0, int pos1) {
  const int n = drafted(a, b);
  // (refused before this round; what this round refuses must not change its rows, which
  // every workgroup counts for itself)
  if (n < pos0 || pos0 + (int)ws.stop[b] > a.D + 1) return RoundRows{0, 0};
  return RoundRows{min(pos1 - 1, n) - pos0 + 1, a.draft ? min(pos1, n) - pos0 : 0};
}

// A row's parts are a wavefront's items.  Up to kListed sequences, the workgroup
// counts the round's rows in order, and cuts them so that the wavefronts share what
// there is to do equally, however few sequences are left; of more, every row has its items, and
// those of rows that are not needed are left out.  Who ends a position's last part
// makes its test.
//
// bf16 rows are bound by HBM (295 MB, the first position of 512 sequences at V =
// 151,936: 64 us, of which reading 53, 5.5 TB/s), fp32 ones by the exponentials in
// double precision (154 MB, the first three of 256 at V = 50,257: 39 us).  Besides, a launch takes about 12 us: the table 4,
// counting 1, the first loads, and at its end the counters and the tests 3 each.
constexpr int kListed = 2048;
template <class TI, bool TABLE>
__global__ void __launch_bounds__(kVerThreads, 4) k_verify_rows(VerifyArgs a, int pos0, int pos1) {
  __shared__ VerTab<TABLE> tab;
  __shared__ union {
    double factors[TABLE ? kTabBinades * 32 : 1];
    uint32_t before[kListed];  // rows of the sequences before each
  } c;
  __shared__ uint32_t wsum[kVerWaves];
  const int tid = threadIdx.x;
  const uint32_t lane = tid & 63;
  const uint32_t w = (uint32_t)__builtin_amdgcn_readfirstlane(tid >> 6);
  const VerWs ws = ver_ws(a);
  const uint32_t W = gridDim.x * kVerWaves;
  uint32_t parts = (uint32_t)a.parts, part_groups = a.part_groups;
  const uint32_t groups = (uint32_t)((a.V + 7) >> 3);
  const bool listed = a.B <= kListed;
  uint64_t items;
  uint32_t all = 0;  // rows of the round
  const uint32_t most = (uint32_t)(pos1 - pos0) * (a.draft ? 2u : 1u);  // rows of a sequence
  constexpr int PER = kListed / kVerThreads;
  uint32_t mine[PER], sum = 0;
  if (listed) {
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int64_t b = (int64_t)tid * PER + k;
      mine[k] = 0;
      if (b < a.B) {
        const RoundRows r = round_rows(a, ws, b, pos0, pos1);
        mine[k] = (uint32_t)(r.targets + r.drafts);
      }
    }
  }
  ver_setup<TABLE, kVerThreads>(tab, c.factors);
  if (listed) {
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const uint32_t rows = mine[k];
      mine[k] = sum;
      sum += rows;
    }
    uint32_t incl = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t x = (uint32_t)__shfl_up((int)incl, o, 64);
      if (lane >= (uint32_t)o) incl += x;
    }
    if (lane == 63) wsum[w] = incl;
    __syncthreads();  // (the table's factors are no longer needed)
    uint32_t at = incl - sum;
    for (uint32_t k = 0; k < w; ++k) at += wsum[k];
#pragma unroll
    for (int k = 0; k < PER; ++k) c.before[tid * PER + k] = at + mine[k];
#pragma unroll
    for (int k = 0; k < kVerWaves; ++k) all += wsum[k];
    __syncthreads();
    // as many parts to a row as give the wavefronts the least to do: whole items, and
    // for each kItemCost of a row besides (the first loads and the record)
    constexpr float kItemCost = 0.03f;
    const uint32_t tiles = (groups + 255) / 256, p = min(lane + 1, (uint32_t)a.parts);  // (64 at most)
    float cost = (float)((all * p + W - 1) / W) * (1.f / (float)p + kItemCost);
    parts = p;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const float x = __shfl_xor(cost, o, 64);
      const uint32_t xp = (uint32_t)__shfl_xor((int)parts, o, 64);
      if (x < cost || (x == cost && xp < parts)) {
        cost = x;
        parts = xp;
      }
    }
    parts = (uint32_t)__builtin_amdgcn_readfirstlane((int)parts);
    part_groups = (tiles + parts - 1) / parts * 256;
    parts = (groups + part_groups - 1) / part_groups;
    items = (uint64_t)all * parts;
  } else {
    items = (uint64_t)a.B * most * parts;
  }
  uint64_t k = (uint64_t)blockIdx.x * kVerWaves + w;
  while (k < items) {
    // up to 64 items, the j-th kept in mind by lane j; then they are announced together
    int64_t my_tr = -1;
    uint32_t my_b = 0;
    int my_pos = 0, my_pair = 0;
    uint32_t held = 0;
    for (; k < items && held < 64; k += W) {
      const uint64_t u = k / parts;
      const uint32_t part = (uint32_t)(k - u * parts);
      uint32_t r;
      int64_t b;
      RoundRows rr;
      if (listed) {
        uint32_t lo = 0, hi = (uint32_t)a.B - 1;  // the last sequence with before <= u
        while (lo < hi) {
          const uint32_t mid = (lo + hi + 1) >> 1;
          if (c.before[mid] <= (uint32_t)u) lo = mid;
          else hi = mid - 1;
        }
        const uint32_t from = c.before[lo];
        const int n = (int)((lo + 1 < (uint32_t)a.B ? c.before[lo + 1] : all) - from);
        // (a target row without a draft row is the last)
        rr = a.draft ? RoundRows{(n + 1) / 2, n / 2} : RoundRows{n, 0};
        b = (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)lo);
        r = (uint32_t)u - from;
      } else {
        b = (int64_t)(u / most);
        r = (uint32_t)(u - (uint64_t)b * most);
        rr = round_rows(a, ws, b, pos0, pos1);
        if (r >= (uint32_t)(rr.targets + rr.drafts)) continue;
      }
      const bool draft = __builtin_amdgcn_readfirstlane(r >= (uint32_t)rr.targets);
      const int pos = __builtin_amdgcn_readfirstlane(pos0 + (int)(draft ? r - rr.targets : r));
      // (refused by now; nothing is while the first items are on their way)
      if (k >= W && pos + (int)ws.stop[b] > a.D + 1) continue;
      const uint32_t g0 = part * part_groups, g1 = min(g0 + part_groups, groups);
      const int64_t tr = target_row(a, b, pos), dr = a.B * (a.D + 1) + draft_row(a, b, pos);
      const VerRec x = part_record<TI, TABLE>(
          draft ? draft_ptr<TI>(a, b, pos) : target_ptr<TI>(a, b, pos), g0, g1, a.V, tab);
      VerRec* rec = ws.rec + (draft ? dr : tr) * a.parts + part;
      if (lane == 0) {
        shared_store(&rec->m, x.m);
        shared_store(&rec->s, x.s);
      }
      if (lane == held) {
        my_tr = tr;
        my_b = (uint32_t)b;
        my_pos = pos;
        my_pair = pos - pos0 < rr.drafts;
      }
      ++held;
    }
    shared_wait();
    uint32_t done = 0;
    if (my_tr >= 0)
      done = 1 + __hip_atomic_fetch_add(&ws.count[my_tr], 1u, __ATOMIC_RELAXED,
                                        __HIP_MEMORY_SCOPE_AGENT);
    // those that ended their position make its test
    uint64_t ends = __ballot(my_tr >= 0 && done == parts * (my_pair ? 2u : 1u));
    while (ends != 0) {
      const int j = first_lane(ends);
      ends &= ends - 1;
      const int64_t b = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)my_b, j);
      const int pos = __builtin_amdgcn_readlane(my_pos, j);
      const bool pair = __builtin_amdgcn_readlane(my_pair, j) != 0;
      const int64_t tr = target_row(a, b, pos), dr = a.B * (a.D + 1) + draft_row(a, b, pos);
      const VerRow rt = row_of_parts(ws.rec + tr * a.parts, (int)parts, tab.p);
      const VerRow rd =
          pair ? row_of_parts(ws.rec + dr * a.parts, (int)parts, tab.p) : VerRow{0.0, 0.0};
      if (lane == 0) {
        ws.row[tr] = rt;
        if (pair) ws.row[dr] = rd;
        if (pos < drafted(a, b)) {
          const uint32_t t = test_token<TI>(a, b, pos, rt, rd, tab.p);
          ws.test[tr] = t;
          // (D + 1 - the first refusal, or 0)
          if (t != kKept)
            __hip_atomic_fetch_max(&ws.stop[b], (uint32_t)(a.D + 1 - pos), __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_AGENT);
        }
      }
    }
  }
}

// ---------------------------------------------------------------- the draw

// The masses that the last token of a sequence is drawn from.
enum Mass : int { kTarget, kResidual, kWithout };  // p; max(p - q, 0); p but for x

template <class TI>
struct DrawRow {
  const char* z;
  const char* y;     // kResidual
  double ps, qs;     // exp(-l) of both
  const VerRow* far;  // the target's and the draft's, in LDS: read where not direct (rare,
                      // and the registers are full) and for the drawn token's log-prob
  int64_t x;         // kWithout: the refused token
  int mass;
  bool direct;       // from exp(z) (as the rows were summed), else from exp(log p)
};

// The masses of a lane's group, in index order.
template <class TI, bool TABLE>
__device__ __forceinline__ void group_masses(const DrawRow<TI>& d, const Group<TI>& z,
                                             const Group<TI>& y, uint32_t g, const VerTab<TABLE>& tab,
                                             double c2, double (&w)[8]) {
  bool rare = false;
  if (d.direct) {
    group_terms<TI, TABLE>(z, tab, c2, rare, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] *= d.ps;
    if (d.mass == kResidual) {
      double v[8];
      group_terms<TI, TABLE>(y, tab, c2, rare, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = fmax(fma(-v[e], d.qs, w[e]), 0.0);
    }
  } else {
    float f[8], h[8];
    group_values<TI>(z, f);
    group_values<TI>(y, h);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      double v = exp_reduced(log_p(f[e], d.far[0]), tab.p, c2);
      if (d.mass == kResidual) v = fmax(v - exp_reduced(log_p(h[e], d.far[1]), tab.p, c2), 0.0);
      w[e] = v;
    }
  }
  if (d.mass == kWithout && (d.x >> 3) == (int64_t)g) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if ((d.x & 7) == e) w[e] = 0.0;
  }
}
// (of group g, read here; groups at or past g1 have none)
template <class TI, bool TABLE>
__device__ __forceinline__ void masses_at(const VerifyArgs& a, const DrawRow<TI>& d, uint32_t g,
                                          uint32_t g1, const VerTab<TABLE>& tab, double c2,
                                          double (&w)[8]) {
  const Group<TI> z = group_load_end<TI>(d.z, g, g1, a.V);
  const Group<TI> y = d.mass == kResidual ? group_load_end<TI>(d.y, g, g1, a.V) : z;
  group_masses<TI, TABLE>(d, z, y, g, tab, c2, w);
}

struct DrawLds {
  double s[kSmpMaxChunks];  // chunk masses
  double p[kVerThreads];    // inclusive prefix of the runs
  double wt[kVerWaves];
  VerRow far[2];
  uint32_t word;
};

// The index drawn from the masses of chunk at.q (chunks of CG groups): the first at
// which they exceed at.r, or (where rounding leaves none) the first or last of
// positive mass.  (One wavefront.)
template <class TI, bool TABLE>
__device__ __forceinline__ int64_t mass_element(const VerifyArgs& a, const DrawRow<TI>& d,
                                                DrawAt at, uint32_t CG, uint32_t groups,
                                                const VerTab<TABLE>& tab, double c2) {
  if (at.q < 0) return -1;
  const uint32_t lane = threadIdx.x & 63;
  const uint32_t c0 = (uint32_t)at.q * CG, c1 = min(c0 + CG, groups);
  double w[8];
  if (at.pick == kCross) {
    double acc = 0.0;
    for (uint32_t g = c0; g < c1; g += 64) {
      masses_at<TI, TABLE>(a, d, g + lane, c1, tab, c2, w);
      const int k = step_crossing(w, at.r, 1.0, acc);
      if (k >= 0) return (int64_t)g * 8 + k;
      if (k == -2) break;
    }
    at.pick = kLast;
  }
  const bool last = at.pick == kLast;
  const uint32_t steps = (c1 - c0 + 63) / 64;
  for (uint32_t k = 0; k < steps; ++k) {
    const uint32_t g = c0 + (last ? steps - 1 - k : k) * 64;
    masses_at<TI, TABLE>(a, d, g + lane, c1, tab, c2, w);
    int ef = -1, eb = -1;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (w[e] > 0.0) {
        if (ef < 0) ef = e;
        eb = e;
      }
    const int vl = last ? last_lane(__ballot(eb >= 0)) : first_lane(__ballot(ef >= 0));
    if (vl >= 0) return (int64_t)(g + vl) * 8 + __builtin_amdgcn_readlane(last ? eb : ef, vl);
  }
  return -1;
}

// The masses of chunks [q0, q1), each by a wavefront; out[q] (shared: by other
// workgroups, too).
template <class TI, bool TABLE>
__device__ __forceinline__ void chunk_masses(const VerifyArgs& a, const DrawRow<TI>& d, uint32_t q0,
                                             uint32_t q1, uint32_t CG, uint32_t groups,
                                             const VerTab<TABLE>& tab, double c2, double* out,
                                             bool shared) {
  constexpr int K = TI::BYTES == 2 ? 4 : 2;  // chunks of one step at a time
  const uint32_t lane = threadIdx.x & 63;
  const uint32_t w = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const uint32_t full = (uint32_t)(a.V >> 3);
  auto put = [&](uint32_t q, double sum) {
    const double all = wave_incl_scan_f64(sum);
    if (lane == 63) {
      if (shared)
        shared_store(out + q, all);
      else
        out[q] = all;
    }
  };
  uint32_t q = q0;
  if (CG == 64) {
    for (; q + K * kVerWaves <= q1 && (q + K * kVerWaves) * 64 <= full; q += K * kVerWaves) {
      const uint32_t qw = q + w * K;
      Group<TI> z[K], y[K];
#pragma unroll
      for (int k = 0; k < K; ++k) {
        z[k] = group_load<TI>(d.z, (qw + k) * 64 + lane);
        y[k] = d.mass == kResidual ? group_load<TI>(d.y, (qw + k) * 64 + lane) : z[k];
      }
#pragma unroll
      for (int k = 0; k < K; ++k) {
        double v[8], sum = 0.0;
        group_masses<TI, TABLE>(d, z[k], y[k], (qw + k) * 64 + lane, tab, c2, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += v[e];
        put(qw + k, sum);
      }
    }
  }
#pragma unroll 1
  for (uint32_t k = q + w; k < q1; k += kVerWaves) {  // the rest one by one
    double sum = 0.0;
    const uint32_t c1 = min(k * CG + CG, groups);
    for (uint32_t g = k * CG; g < c1; g += 64) {
      double v[8];
      masses_at<TI, TABLE>(a, d, g + lane, c1, tab, c2, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += v[e];
    }
    put(k, sum);
  }
}

// A sequence's tokens: the kept ones, then the draw.  The row that it is drawn from
// (for a residual, the draft's too) is read again, as its masses need both rows'
// sums: 237 MB in 65 us at 512 sequences of 8 drafts, V = 151,936 (3.6 TB/s: a
// workgroup to a sequence, whose loads of a step do not overlap the sums of the step
// before); 23 us at 64 of 5, of which the table is 4 and the last workgroup of a
// sequence 6.  Item k: part k % draw_parts of
// the row that sequence k / draw_parts is drawn from; whoever ends a sequence's
// last part draws.
template <class TI, bool TABLE>
__global__ void __launch_bounds__(kVerThreads, 4) k_verify_draw(VerifyArgs a) {
  __shared__ VerTab<TABLE> tab;
  __shared__ DrawLds c;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const VerWs ws = ver_ws(a);
  const uint32_t groups = (uint32_t)((a.V + 7) >> 3);
  const uint32_t nchunk = (uint32_t)a.nchunk, CG = 64u * (uint32_t)a.chunk_steps;
  const int parts = a.draw_parts;
  const double c2 = c2_reg();
  static_assert(kTabBinades * 32 <= kSmpMaxChunks, "the table's factors fit the masses");
  // (the first item's words are on their way during the setup)
  int n = drafted(a, blockIdx.x / parts);
  uint32_t stop = ws.stop[blockIdx.x / parts];
  ver_setup<TABLE, kVerThreads>(tab, c.s);
  for (int64_t k = blockIdx.x; k < a.B * parts; k += gridDim.x) {
    const int64_t b = k / parts;
    const uint32_t part = (uint32_t)(k - b * parts);
    int32_t* ids = a.ids_out + b * (a.D + 1);
    float* logp = a.logp ? a.logp + b * (a.D + 1) : nullptr;
    const bool masked = a.mask && a.mask[b] == 0;
    if (k != blockIdx.x) {
      n = drafted(a, b);
      stop = ws.stop[b];
    }
    // the first token that is not kept
    const uint32_t st = n < 0 ? 0 : stop;
    const int kept = n < 0 ? 0 : st ? a.D + 1 - (int)st : n;
    const uint32_t test = n < 0 ? (uint32_t)kBad : st ? ws.test[b * (a.D + 1) + kept] : (uint32_t)kKept;
    const float u = a.u[b * (a.D + 1) + a.D];
    DrawRow<TI> d{};
    VerRow rt{__builtin_nan(""), 0.0}, rd{0.0, 0.0};
    if (!masked && test != kBad) {
      rt = ws.row[target_row(a, b, kept)];
      d.z = target_ptr<TI>(a, b, kept);
      d.mass = kTarget;
      if (test == kRefused) {
        d.mass = a.draft ? kResidual : kWithout;
        d.x = a.ids[b * a.D + kept];
        if (a.draft) {
          rd = ws.row[a.B * (a.D + 1) + draft_row(a, b, kept)];
          d.y = draft_ptr<TI>(a, b, kept);
        }
      }
      d.ps = exp(-rt.l);
      d.qs = exp(-rd.l);
      // (both rows summed as exp(z): no logit at or past kVerTop, and no tiny sum)
      d.direct = rt.m == 0.0 && rd.m == 0.0;
      d.far = c.far;
      if (tid == 0) {  // (the item before is done with c)
        c.far[0] = rt;
        c.far[1] = rd;
      }
      if (!d.direct) __syncthreads();  // (the same in every lane)
    }
    const bool draws = rt.l == rt.l && u >= 0.f && u < 1.f;
    if (parts > 1) {
      if (draws) {
        const uint32_t per = (nchunk + parts - 1) / parts;
        const uint32_t q0 = min(part * per, nchunk), q1 = min(q0 + per, nchunk);
        chunk_masses<TI, TABLE>(a, d, q0, q1, CG, groups, tab, c2,
                                ws.mass + b * (int64_t)nchunk, true);
        shared_wait();
      }
      __syncthreads();
      if (tid == 0)
        c.word = __hip_atomic_fetch_add(&ws.done[b], 1u, __ATOMIC_RELAXED,
                                        __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)parts - 1;
      __syncthreads();
      const bool last = c.word != 0u;
      __syncthreads();
      if (!last) continue;
    }
    for (int i = tid; i <= a.D; i += kVerThreads) {
      const bool mine = !masked && i < kept;
      const int32_t x = mine ? a.ids[b * a.D + i] : -1;
      if (i != kept || masked || !draws) ids[i] = x;
      if (logp && (i != kept || masked || !draws))
        logp[i] = mine ? (float)log_p(load_elem<TI>(target_ptr<TI>(a, b, i), x),
                                      ws.row[target_row(a, b, i)])
                       : (i == kept && !masked ? __builtin_nanf("") : 0.f);
    }
    if (tid == 0) a.accepted[b] = kept;
    if (masked || !draws) continue;
    double S = 0.0;
    bool mine = parts == 1;  // this workgroup makes the masses
    for (;;) {
      if (mine)
        chunk_masses<TI, TABLE>(a, d, 0, nchunk, CG, groups, tab, c2, c.s, false);
      else
        for (uint32_t q = tid; q < nchunk; q += kVerThreads)
          c.s[q] = shared_load(ws.mass + b * (int64_t)nchunk + q);
      __syncthreads();
      const uint32_t C = (nchunk + kVerThreads - 1) / kVerThreads;
      const uint32_t r0 = min((uint32_t)tid * C, nchunk), r1 = min(r0 + C, nchunk);
      double run = 0.0;
      for (uint32_t q = r0; q < r1; ++q) run += c.s[q];
      const double incl = wave_incl_scan_f64(run);
      if (lane == 63) c.wt[w] = incl;
      __syncthreads();
      double before = 0.0;
      for (int i = 0; i < w; ++i) before += c.wt[i];
      c.p[tid] = before + incl;
      S = 0.0;
#pragma unroll
      for (int i = 0; i < kVerWaves; ++i) S += c.wt[i];
      __syncthreads();
      // p(x) < q(x) leaves a residual; where rounding hides it the draw is from p
      if (S > 0.0 || d.mass == kTarget) break;
      d.mass = kTarget;
      d.direct = c.far[0].m == 0.0;
      mine = true;
    }
    if (w == 0) {
      const uint32_t C = (nchunk + kVerThreads - 1) / kVerThreads;
      const DrawAt at = smp_locate<kVerThreads>(c, nchunk, C, (double)u * S, S);
      const int64_t id = mass_element<TI, TABLE>(a, d, at, CG, groups, tab, c2);
      if (lane == 0) {
        ids[kept] = (int32_t)id;
        if (logp)
          logp[kept] = id >= 0 ? (float)log_p(load_elem<TI>(d.z, id), c.far[0])
                               : __builtin_nanf("");
      }
    }
    __syncthreads();  // (the masses are used until here)
  }
}

template <class TI, bool TABLE>
hipError_t launch_verify_t(const VerifyArgs& a, hipStream_t stream) {
  const int64_t words = a.B * (2 * (a.D + 1) + 2);
  const int64_t R = a.B * (2 * a.D + 1);
  uint32_t* first = (uint32_t*)((char*)a.ws + R * sizeof(VerRow) +
                                R * a.parts * sizeof(VerRec) +
                                (a.draw_parts > 1 ? a.B * (int64_t)a.nchunk * sizeof(double) : 0));
  hipLaunchKernelGGL(k_verify_clear, dim3((unsigned)min((words + 255) / 256, (int64_t)64)), dim3(256),
                     0, stream, first, words);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  for (int pos = 0, many = a.round; pos <= a.D; pos += many, many *= 2) {
    if (many > a.D + 1 - pos) many = a.D + 1 - pos;
    const int64_t items = a.B * a.parts * many * (a.draft ? 2 : 1);  // at most
    hipLaunchKernelGGL((k_verify_rows<TI, TABLE>),
                       dim3((unsigned)min((items + kVerWaves - 1) / kVerWaves, (int64_t)kVerGroups)),
                       dim3(kVerThreads), 0, stream, a, pos, pos + many);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((k_verify_draw<TI, TABLE>),
                     dim3((unsigned)min(a.B * a.draw_parts, (int64_t)kVerGroups)),
                     dim3(kVerThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_verify(const VerifyArgs& a, int in_dt, hipStream_t stream) {
  if (in_dt == F32) return launch_verify_t<InF32, false>(a, stream);
  // The table is set up by each workgroup (a few us); few rows are summed without it.
  return a.table ? launch_verify_t<InBf16, true>(a, stream)
                 : launch_verify_t<InBf16, false>(a, stream);
}

}  // namespace opd
