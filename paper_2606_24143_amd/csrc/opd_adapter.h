// Low-rank adapters of many requests at once, beside a projection that all share
// (the output head's rows of logits, or any other), and their gradients.  With
// a [G, r, H] and b [G, r, O], both rows of the long axis, and token n of adapter g:
//   t = x a_g^T (r numbers),  out = y + s_g t b_g
//   u = dy b_g^T,             dx = s_g u a_g (+ the shared projection's),
//   da_g = s_g sum_n u_n^T x_n,  db_g = s_g sum_n t_n^T dy_n
// Three products on the matrix cores carry both directions: tokens times the rows
// of an adapter (k_low: t and u), those r numbers times the rows (k_expand: out
// and dx), and summed over an adapter's tokens (k_outer: da and db).  All read
// their operands from memory in the order in which they lie there, 16 bytes a lane, and
// none needs LDS for them: the sum's index may run in any order, and where
// a product needs a lane's eight values to lie along tokens or ranks instead, the lane
// loads an 8 by 8 block and transposes it in its registers.
// Sums are fp32; beside bf16 operands t and u pass to the second product as three bf16 parts
// (2^-25 of them, as good as fp32, also where results cancel).  fp32 operands take the fp32
// matrix instructions, exact products throughout.
#pragma once

#include "opd_device.h"
#include "opd_group.h"
#include "opd_model.h"
#include "opd_piece.h"

namespace opd {
namespace {

typedef __bf16 BFrag __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------- tokens by adapter

constexpr int kAdKeys = 1024;
struct PlanLds {
  GroupLds<kAdKeys> group;
  uint32_t tile[kAdKeys + 1];
};

// One workgroup: tokens sorted by adapter (key G: none, G + 1: an id outside [0, G)),
// and tiles of kAdTile tokens of one key.
__global__ void __launch_bounds__(kGroupThreads) k_adapt_plan(AdaptArgs a) {
  __shared__ PlanLds sh;
  const int32_t G = a.G;
  const int32_t* ids = a.ids;
  const int count = G + 2;
  uint32_t end;
  const uint32_t first = group_tokens<kAdKeys, false>(
      a.N, 0, count,
      [=](int64_t n) {
        const int32_t id = ids[n];
        return id == -1 ? G : (uint32_t)id < (uint32_t)G ? id : G + 1;
      },
      a.perm, sh.group, end);
  // (the first places once more, for the counts)
  __syncthreads();
  uint32_t* const place = &sh.group.at[0][0];
  if ((int)threadIdx.x < count) {
    place[threadIdx.x] = first;
    if (a.start) a.start[threadIdx.x] = (int32_t)first;
  }
  if ((int)threadIdx.x == count) {
    place[count] = end;
    if (a.start) a.start[count] = (int32_t)end;
  }
  __syncthreads();
  const uint32_t tokens =
      (int)threadIdx.x < count ? place[threadIdx.x + 1] - place[threadIdx.x] : 0u;
  const uint32_t mine = (tokens + kAdTile - 1) / kAdTile;
  uint32_t total;
  const uint32_t tile = block_excl_scan(mine, sh.group.sums, total);
  if ((int)threadIdx.x < count) sh.tile[threadIdx.x] = tile;
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < (uint32_t)a.max_tiles; i += kGroupThreads) {
    AdTile t = {0, 0, 0, 0};
    if (i < total) {
      // the last key whose tiles begin at or before i and that has some
      int lo = 0, hi = count - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (sh.tile[mid] <= i)
          lo = mid;
        else
          hi = mid - 1;
      }
      const uint32_t at = place[lo] + (i - sh.tile[lo]) * kAdTile;
      t.key = lo;
      t.pos = (int32_t)at;
      t.count = (int32_t)min((uint32_t)kAdTile, place[lo + 1] - at);
    }
    a.tiles[i] = t;
  }
}

// The same for up to kAdFew tokens, by a wavefront of each workgroup that needs them: perm
// [kAdFew] and tiles [kAdFew] (one to a key) in LDS; the number of tiles.  4,096 columns, the
// call on the GPU: 64 tokens of 32 adapters 9.6 us, 13.8 with a launch before for the tiles; 1
// token 6.9 and 11.3.
__device__ __forceinline__ int plan_few(const int32_t* ids, int N, int32_t G, int32_t* perm,
                                        AdTile* tiles) {
  const int lane = threadIdx.x & 63;
  const int32_t id = ids[min(lane, N - 1)];
  const int32_t key = id == -1 ? G : (uint32_t)id < (uint32_t)G ? id : G + 1;
  const uint64_t in = N == 64 ? ~0ull : (1ull << N) - 1;
  // lanes of smaller keys, and of this one, by the keys' bits
  uint64_t less = 0, same = in;
  for (int bit = 31 - __clz(G + 1); bit >= 0; --bit) {
    const int32_t mine = -(key >> bit & 1);  // (all bits, or none)
    const uint64_t b = __ballot(mine != 0);
    less |= same & ~b & (uint64_t)(int64_t)mine;
    same &= ~(b ^ (uint64_t)(int64_t)mine);
  }
  const int count = __popcll(same), place = __popcll(less);
  const bool first = lane < N && lane == __ffsll((long long)same) - 1;
  const uint64_t firsts = __ballot(first);
  const int all = __popcll(firsts), tile = __popcll(less & firsts);
  if (lane < N) perm[place + __popcll(same & ((1ull << lane) - 1))] = lane;
  if (first) tiles[tile] = AdTile{key, place, count, 0};
  return all;
}

// ---------------------------------------------------------------- loads

// Columns at or past `end` of those from c on become 0.
template <class T>
__device__ __forceinline__ u32x4 cut16(u32x4 r, int64_t c, int64_t end) {
  constexpr int E = 16 / T::BYTES;
  const int valid = end - c > E ? E : end - c < 0 ? 0 : (int)(end - c);
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    if constexpr (T::BYTES == 2) {
      const uint32_t keep =
          (2 * d < valid ? 0x0000FFFFu : 0u) | (2 * d + 1 < valid ? 0xFFFF0000u : 0u);
      r[d] &= keep;
    } else {
      r[d] = d < valid ? r[d] : 0u;
    }
  }
  return r;
}
__device__ __forceinline__ f32x4 cut4(f32x4 f, int64_t c, int64_t end) {
#pragma unroll
  for (int e = 0; e < 4; ++e) f[e] = c + e < end ? f[e] : 0.f;
  return f;
}

__device__ __forceinline__ f32x4 mma_bf16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(BFrag, a),
                                                 __builtin_bit_cast(BFrag, b), c, 0, 0, 0);
}
// (16 ranks: a lane's four)
__device__ __forceinline__ f32x4 mma_bf16_16(u32x2 a, u32x2 b, f32x4 c) {
  typedef short S4 __attribute__((ext_vector_type(4)));
  return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(S4, a),
                                                   __builtin_bit_cast(S4, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma_f32(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// A number as bf16 parts that add up to it (one to 2^-9, two to 2^-17, three to 2^-25 of it); one
// that is not finite in bf16 is its first part.
constexpr int kAdTerms = 3;
__device__ __forceinline__ void split_bf16(float f, uint16_t (&p)[kAdTerms]) {
#pragma unroll
  for (int i = 0; i < kAdTerms; ++i) {
    const __bf16 h = (__bf16)f;
    p[i] = __builtin_bit_cast(uint16_t, h);
    const float r = f - (float)h;
    f = (p[i] & 0x7F80u) == 0x7F80u ? 0.f : r;
  }
}

// The r numbers of a token from what k_low left (or the caller kept): sums over
// `splits` parts of the long axis.
__device__ __forceinline__ float low_value(const LowRef& t, int64_t token, int c) {
  float f = 0.f;
  if (c < t.r) {
    const float* p = t.p + token * t.ld + c;
    f = p[0];
    for (int s = 1; s < t.splits; ++s) f += p[(int64_t)s * t.stride];
  }
  return f;
}

// ---------------------------------------------------------------- tokens times the rows

// One workgroup to 16 MT tokens of an adapter and a part of the long axis: its waves
// take steps of 64 (bf16) or 32 (fp32) columns in turn, the next ones on their way meanwhile,
// and their sums are added in order.  A lane's operands lie along a row, and its
// neighbours' in other rows: loaded so, an instruction touches 16 lines 16 bytes at a time,
// which took 10 us more for 8,192 tokens by 4,096 columns and 32 ranks than rows read as they
// lie and turned in LDS, a part of it to each wave: 23.2 us, 20 where nothing has just been
// written (reading the tokens alone takes 17.5).  RT: ranks / 16.
constexpr int kLowThreads = 512;
constexpr int kLowWaves = kLowThreads / 64;

// ROWS rows of a step (128 bytes each, or 64), by a wave: as they lie in memory, and in LDS,
// where the 16-byte pieces of a row are rotated so that the same piece of eight rows
// lies in different banks.
template <int ROWS, int ROW_BYTES>
struct Staged {
  static constexpr int P = ROW_BYTES / 16, PER = 64 / P;  // pieces of a row, rows of an instruction
  static constexpr int N = ROWS / PER;
  u32x4 v[N];
  static __device__ __forceinline__ int row(int i) { return i * PER + (threadIdx.x & 63) / P; }
  static __device__ __forceinline__ int piece() { return (threadIdx.x & 63) % P; }
  static __device__ __forceinline__ int slot(int row, int p) { return row * P + (p ^ (row & (P - 1))); }
  __device__ __forceinline__ void put(u32x4* lds) const {
#pragma unroll
    for (int i = 0; i < N; ++i) lds[slot(row(i), piece())] = v[i];
  }
};

template <class TX, class TW, int RT, int MT>
__global__ void __launch_bounds__(kLowThreads, 2) k_low(LowPair pair) {
  const bool second = (int)blockIdx.y >= pair.a[0].splits;
  const LowArgs& a = pair.a[second];
  const int split = (int)blockIdx.y - (second ? pair.a[0].splits : 0);
  constexpr bool BF = TX::BYTES == 2 && TW::BYTES == 2;
  constexpr int STEP = BF ? 64 : 32;
  typedef std::conditional_t<BF, u32x4, f32x4> V;
  typedef Staged<16 * MT, STEP * TX::BYTES> SX;
  typedef Staged<16 * RT, STEP * TW::BYTES> SW;
  constexpr int XV = 16 * MT * SX::P, WV = 16 * RT * SW::P;  // 16-byte vectors of a wave's step
  constexpr int SUM = 16 * MT * (RT * 16 + 1);
  constexpr int AHEAD = RT <= 2 ? 3 : RT <= 4 ? 2 : 1;  // steps on their way
  constexpr int EACH = (XV + WV) * 4 > SUM ? (XV + WV) * 4 : (SUM + 3) / 4 * 4;
  __shared__ __align__(16) float lds[kLowWaves][EACH];
  __shared__ int32_t tokens[16 * MT];
  constexpr int SUBS = kAdTile / (16 * MT);
  const int sub = blockIdx.x % SUBS * (16 * MT);
  AdTile tile;
  if (a.ids) {
    __shared__ struct {
      int32_t perm[kAdFew];
      AdTile tiles[kAdFew];
      int all;
    } few;
    if (threadIdx.x < 64) few.all = plan_few(a.ids, a.N, a.G, few.perm, few.tiles);
    __syncthreads();
    if (blockIdx.x == 0 && blockIdx.y == 0) {  // for the second product
      if ((int)threadIdx.x < a.N) a.perm[threadIdx.x] = few.perm[threadIdx.x];
      if ((int)threadIdx.x < (int)a.max_tiles)
        a.tiles[threadIdx.x] =
            (int)threadIdx.x < few.all ? few.tiles[threadIdx.x] : AdTile{0, 0, 0, 0};
    }
    if ((int)(blockIdx.x / SUBS) >= few.all) return;
    tile = few.tiles[blockIdx.x / SUBS];
    if (sub >= tile.count || tile.key >= a.G) return;
    if (threadIdx.x < 16 * MT)
      tokens[threadIdx.x] = few.perm[tile.pos + min(sub + (int)threadIdx.x, tile.count - 1)];
  } else {
    tile = a.tiles[blockIdx.x / SUBS];
    if (sub >= tile.count || tile.key >= a.G) return;
    if (threadIdx.x < 16 * MT)
      tokens[threadIdx.x] = a.perm[tile.pos + min(sub + (int)threadIdx.x, tile.count - 1)];
  }
  __syncthreads();
  const int lane = threadIdx.x & 63, m = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int count = min(16 * MT, tile.count - sub);
  u32x4* const lx = (u32x4*)lds[wave];
  u32x4* const lw = lx + XV;
  const char* x[SX::N];
#pragma unroll
  for (int i = 0; i < SX::N; ++i)
    x[i] = (const char*)a.x + (int64_t)tokens[SX::row(i)] * a.ldx * TX::BYTES;
  const char* w = (const char*)a.w + (int64_t)tile.key * a.r * a.ldw * TW::BYTES;
  const uint32_t ldw = (uint32_t)a.ldw * TW::BYTES;
  f32x4 acc[MT][RT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
#pragma unroll
    for (int t = 0; t < RT; ++t) acc[i][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int64_t d0 = (int64_t)split * a.span;
  const int64_t d1 = d0 + a.span < a.D ? d0 + a.span : a.D;
  struct Step {
    SX x;
    SW w;
  };
  // (No load depends on a condition, since the compiler waits for all where it can't count
  // them: pieces past the end are the last one again, ranks past r the last rank.)
  uint32_t row[SW::N];
#pragma unroll
  for (int i = 0; i < SW::N; ++i) row[i] = (uint32_t)min(SW::row(i), a.r - 1) * ldw;
  auto load = [&](Step& s, int64_t d) {
    const int64_t dx = piece_column<16 / TX::BYTES>(d, SX::piece(), d1) * TX::BYTES;
    const int64_t dw = piece_column<16 / TW::BYTES>(d, SW::piece(), d1) * TW::BYTES;
#pragma unroll
    for (int i = 0; i < SX::N; ++i) s.x.v[i] = *(const u32x4*)(x[i] + dx);
#pragma unroll
    for (int i = 0; i < SW::N; ++i) s.w.v[i] = *(const u32x4*)(w + dw + row[i]);
  };
  // Two instructions' worth of both operands: columns d + 16 q .. + 16 (bf16) or d + 8 q ..
  // + 8, of row m.
  auto add = [&](int64_t d) {
    if (d >= d1) return;
    V xv[MT][2], wv[RT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
        xv[i][h] = __builtin_bit_cast(V, lx[SX::slot(16 * i + m, 2 * q + h)]);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        if constexpr (SW::P == 8) {
          wv[t][h] = __builtin_bit_cast(V, lw[SW::slot(16 * t + m, 2 * q + h)]);
        } else {
          const u32x4 v = lw[SW::slot(16 * t + m, q)];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            wv[t][h][e] = __uint_as_float(e & 1 ? v[2 * h + e / 2] & 0xFFFF0000u
                                                : v[2 * h + e / 2] << 16);
        }
      }
    }
    if (d + STEP > d1) {  // (what lies past the row's end may be anything)
      const int64_t c = d + STEP / 4 * q;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          if constexpr (BF)
            xv[i][h] = cut16<TX>(xv[i][h], c + 8 * h, d1);
          else
            xv[i][h] = cut4(xv[i][h], c + 4 * h, d1);
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          if constexpr (BF)
            wv[t][h] = cut16<TW>(wv[t][h], c + 8 * h, d1);
          else
            wv[t][h] = cut4(wv[t][h], c + 4 * h, d1);
        }
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (BF) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
#pragma unroll
          for (int i = 0; i < MT; ++i) acc[i][t] = mma_bf16(xv[i][h], wv[t][h], acc[i][t]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
          for (int t = 0; t < RT; ++t) {
#pragma unroll
            for (int i = 0; i < MT; ++i) acc[i][t] = mma_f32(xv[i][h][e], wv[t][h][e], acc[i][t]);
          }
        }
      }
    }
  };
  // The rows lie a multiple of the memory channels' period apart, as a rule: workgroups that
  // ran along them side by side would all ask the same channels.  So each starts at
  // another step, and goes round.
  constexpr int NEXT = kLowWaves * STEP;
  const int steps = (int)((d1 - d0 + NEXT - 1) / NEXT);
  int at = (int)(blockIdx.x % (uint32_t)steps), to = at;
  auto column = [&](int& at) {
    const int64_t d = d0 + (int64_t)at * NEXT + wave * STEP;
    at = at + 1 == steps ? 0 : at + 1;
    return d;
  };
  Step s[AHEAD];
  // (Lanes read what others wrote, and write over what others read.  A wave's LDS accesses are
  // done in order; this keeps the compiler to that order.  No wait comes of it, and loads from
  // memory pass.)
  auto ordered = []() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
  };
  auto use = [&](Step& s) {
    ordered();
    s.x.put(lx);
    s.w.put(lw);
    ordered();
  };
#pragma unroll
  for (int j = 0; j < AHEAD; ++j) load(s[j], column(to));
  int left = steps;
#pragma unroll 1
  for (; left > AHEAD; left -= AHEAD) {
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      use(s[j]);
      load(s[j], column(to));
      add(column(at));
    }
  }
#pragma unroll
  for (int j = 0; j < AHEAD; ++j) {
    if (j >= left) continue;
    use(s[j]);
    add(column(at));
  }
  __syncthreads();
  auto sums = [&](int v, int n, int c) -> float& { return lds[v][n * (RT * 16 + 1) + c]; };
#pragma unroll
  for (int i = 0; i < MT; ++i) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
      for (int e = 0; e < 4; ++e) sums(wave, 16 * i + 4 * q + e, 16 * t + m) = acc[i][t][e];
    }
  }
  __syncthreads();
  float* out = a.out + (int64_t)split * a.stride;
  for (int i = threadIdx.x; i < count * a.r; i += kLowThreads) {
    const int n = i / a.r, c = i % a.r;
    float f = sums(0, n, c);
#pragma unroll
    for (int v = 1; v < kLowWaves; ++v) f += sums(v, n, c);
    out[(int64_t)tokens[n] * a.ldo + c] = f;
  }
}

// ---------------------------------------------------------------- the r numbers times the rows

constexpr int kExpThreads = 256;
constexpr int kExpWaves = kExpThreads / 64;

// The first `valid` elements of a vector of a row.
template <class T>
__device__ __forceinline__ void store_end(char* p, u32x4 x, int64_t valid) {
  constexpr int S = 16 / T::BYTES;
  if (valid >= S) {
    *(u32x4*)p = x;
    return;
  }
#pragma unroll
  for (int e = 0; e < S; ++e) {
    if (e >= valid) continue;
    if constexpr (T::BYTES == 2)
      ((uint16_t*)p)[e] = (uint16_t)(x[e / 2] >> (16 * (e & 1)));
    else
      ((uint32_t*)p)[e] = x[e];
  }
}
template <class T, int E>
__device__ __forceinline__ void store_values(char* row, int64_t c, int64_t end, const float (&f)[E]) {
  if (c + E <= end) {
    if constexpr (T::BYTES == 2) {
      static_assert(E == 8, "16 bytes");
      *(u32x4*)(row + c * 2) = u32x4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]),
                                     pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
    } else {
#pragma unroll
      for (int v = 0; v < E / 4; ++v)
        *(f32x4*)(row + c * 4 + 16 * v) =
            f32x4{f[4 * v], f[4 * v + 1], f[4 * v + 2], f[4 * v + 3]};
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (c + e >= end) continue;
      if constexpr (T::BYTES == 2)
        ((__bf16*)row)[c + e] = (__bf16)f[e];
      else
        ((float*)row)[c + e] = f[e];
    }
  }
}

// One workgroup to a tile of up to kAdTile tokens of an adapter and every a.per-th group of
// 4 waves' columns (128 each, or 64 of fp32 rows): a wave keeps its columns of the
// adapter in registers and passes over the tokens, 16 at a time.  The shared projection's
// values are what the sums start from, and become the results in place.  The next 16
// tokens' are on their way meanwhile (no load in a loop depends on a condition, since the
// compiler waits for all where it can't count them); where there are no more than 16, of up
// to 16 ranks, the next columns of the adapter too.
// 8,192 tokens by 4,096 columns and 32 ranks: 34.9 us, 28 at a copy's rate.  The shared
// projection's values and the results pass the caches: kept there, they drain while the next
// call's k_low reads, which then takes 31.8 us instead of 23.2 (and this 33.3).  Two parts of t
// instead of three would save 0.3 us of it, 2 of 90 with 64 ranks, 10 of 141 with 128.
// KL: ranks of a lane's operand (bf16: 4 or 8); RB: of 4 KL ranks each; READ: there is a base.
template <class TW, class TY, int KL, int RB, bool READ>
__global__ void __launch_bounds__(kExpThreads, KL * RB <= 8 ? 4 : 2) k_expand(ExpandArgs a) {
  constexpr bool BF = TW::BYTES == 2;
  constexpr int E = BF ? 8 : 4;          // columns of a lane
  constexpr int S = 16 / TY::BYTES;      // of a vector of the result
  constexpr int TERMS = kAdTerms;
  constexpr int K = 4 * KL * RB;         // ranks
  constexpr int KP = BF ? K + 8 : K + 4; // (padded: lanes of a read spread over the banks)
  constexpr int WV = KL * RB;            // 16-byte vectors of the adapter to a lane
  __shared__ __align__(16) uint16_t part[BF ? TERMS : 1][BF ? kAdTile : 1][KP];
  __shared__ float wide[BF ? 1 : kAdTile][BF ? 1 : KP];
  __shared__ int32_t tokens[kAdTile];
  // (columns first: workgroups side by side read whole rows)
  const uint32_t chunk = blockIdx.x % a.per;
  const AdTile tile = a.tiles[blockIdx.x / a.per];
  if (tile.count == 0) return;
  const int lane = threadIdx.x & 63, m = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t* perm = a.perm + tile.pos;
  const int64_t span = kExpWaves * 16 * E, step = a.per * span;
  int64_t c0 = (int64_t)chunk * span + wave * (16 * E);
  if ((int)threadIdx.x < kAdTile)
    tokens[threadIdx.x] = perm[min((int)threadIdx.x, tile.count - 1)];
  typedef u32x4 Y[4][E / S];
  // columns c0 + m E .. of the wave's, of tokens n0 + 4 q + i: a token's results lie side by
  // side in 16 lanes.  (Past the row's end: its last vector again.)
  const int64_t end = (a.D - 1) / S * S;
  auto load_y = [&](int64_t c0, int n0, Y& y) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const char* row = (const char*)a.base + (int64_t)tokens[n0 + 4 * q + i] * a.ldb * TY::BYTES;
#pragma unroll
      for (int h = 0; h < E / S; ++h) {
        if constexpr (READ)
          y[i][h] = __builtin_nontemporal_load(
              (const u32x4*)(row + min(c0 + m * E + S * h, end) * TY::BYTES));
        else
          y[i][h] = u32x4{0, 0, 0, 0};
      }
    }
  };
  auto store_y = [&](int64_t c0, int n0, const Y& y) {
    const bool whole = c0 + 16 * E <= a.D;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = n0 + 4 * q + i;
      if (n >= tile.count) continue;
      char* row = (char*)a.out + (int64_t)tokens[n] * a.ldo * TY::BYTES + (c0 + m * E) * TY::BYTES;
#pragma unroll
      for (int h = 0; h < E / S; ++h) {
        if (whole)
          __builtin_nontemporal_store(y[i][h], (u32x4*)(row + 16 * h));
        else
          store_end<TY>(row + 16 * h, y[i][h], a.D - (c0 + m * E + S * h));
      }
    }
  };
  if (tile.key >= a.G) {  // no adapter (the base as it is), or a bad id (NaN)
    if (a.low_out && chunk == 0) {
      for (int i = threadIdx.x; i < tile.count * a.r; i += kExpThreads)
        a.low_out[(int64_t)perm[i / a.r] * a.r + i % a.r] =
            tile.key == a.G ? 0.f : __builtin_nanf("");
    }
    if (tile.key == a.G && a.base == a.out) return;  // in place
    __syncthreads();
    for (; c0 < a.D; c0 += step) {
#pragma unroll 1
      for (int n0 = 0; n0 < tile.count; n0 += 16) {
        Y y;
        load_y(c0, n0, y);
        constexpr uint32_t nan = TY::BYTES == 2 ? 0x7FC07FC0u : 0x7FC00000u;
        if (tile.key > a.G) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int h = 0; h < E / S; ++h) y[i][h] = u32x4{nan, nan, nan, nan};
          }
        }
        store_y(c0, n0, y);
      }
    }
    return;
  }
  const char* w = (const char*)a.w + (int64_t)tile.key * a.r * a.ldw * TW::BYTES;
  const uint32_t ldw = (uint32_t)a.ldw * TW::BYTES;
  const int64_t wend = (a.D - 1) / E * E;
  // a wave's columns of the adapter, as they lie, 4 KL ranks at a time: ranks KL q + i (fp32:
  // 4 i + q; past r: the last one again)
  typedef u32x4 W[KL];
  auto rank = [&](int k, int i) { return 4 * KL * k + (BF ? KL * q + i : 4 * i + q); };
  auto load_w = [&](int64_t c0, int k, W& v) {
    const uint32_t c = (uint32_t)min(c0 + m * E, wend) * TW::BYTES;
#pragma unroll
    for (int i = 0; i < KL; ++i)
      v[i] = *(const u32x4*)(w + ((uint32_t)min(rank(k, i), a.r - 1) * ldw + c));
  };
  // the operand: for column j of a lane, its KL ranks
  struct Operand {
    uint32_t b[BF ? RB : 1][8][BF ? KL / 2 : 1];
    f32x4 f[BF ? 1 : WV];
  };
  auto operand = [&](int k, W& v, Operand& o) {
    if (a.r < K) {
#pragma unroll
      for (int i = 0; i < KL; ++i) {
#pragma unroll
        for (int d = 0; d < 4; ++d) v[i][d] = rank(k, i) < a.r ? v[i][d] : 0u;
      }
    }
    if constexpr (BF) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
#pragma unroll
        for (int d = 0; d < KL / 2; ++d)
          o.b[k][j][d] = __builtin_amdgcn_perm(v[2 * d + 1][j / 2], v[2 * d][j / 2],
                                               j & 1 ? 0x07060302u : 0x05040100u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < KL; ++i) o.f[KL * k + i] = __builtin_bit_cast(f32x4, v[i]);
    }
  };
  auto product = [&](const Operand& o, int n0, int j, f32x4 acc) {
    if constexpr (BF) {
#pragma unroll
      for (int k = 0; k < RB; ++k) {
#pragma unroll
        for (int t = TERMS - 1; t >= 0; --t) {
          const uint16_t* low = &part[t][n0 + m][4 * KL * k + KL * q];
          if constexpr (KL == 8)
            acc = mma_bf16(*(const u32x4*)low,
                           u32x4{o.b[k][j][0], o.b[k][j][1], o.b[k][j][2], o.b[k][j][3]}, acc);
          else
            acc = mma_bf16_16(*(const u32x2*)low, u32x2{o.b[k][j][0], o.b[k][j][1]}, acc);
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < WV; ++k) acc = mma_f32(wide[n0 + m][4 * k + q], o.f[k][j], acc);
    }
    return acc;
  };
  auto update = [&](const Operand& o, int n0, Y& y) {
    if constexpr (TY::BYTES == 2) {
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        f32x4 lo, hi;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          lo[i] = __uint_as_float(y[i][0][d] << 16);
          hi[i] = __uint_as_float(y[i][0][d] & 0xFFFF0000u);
        }
        lo = product(o, n0, 2 * d, lo);
        hi = product(o, n0, 2 * d + 1, hi);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i][0][d] = pack_bf16x2(lo[i], hi[i]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j) {
        f32x4 acc;
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = __uint_as_float(y[i][j / 4][j % 4]);
        acc = product(o, n0, j, acc);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i][j / 4][j % 4] = __float_as_uint(acc[i]);
      }
    }
  };
  W v;
  load_w(c0, 0, v);
  const float scale = a.scales ? a.scales[tile.key] : 1.f;
  for (int i = threadIdx.x; i < kAdTile * K; i += kExpThreads) {
    const int n = i / K, k = i % K;
    float f = 0.f;
    if (n < tile.count && k < a.r) {
      const int64_t token = perm[n];
      f = low_value(a.low, token, k);
      if (a.low_out && chunk == 0) a.low_out[token * a.r + k] = f;
      f *= scale;
    }
    if constexpr (BF) {
      uint16_t p[TERMS];
      split_bf16(f, p);
#pragma unroll
      for (int t = 0; t < TERMS; ++t) part[t][n][k] = p[t];
    } else {
      wide[n][k] = f;
    }
  }
  __syncthreads();
  Y y, z;
  Operand o;
  if (KL == 4 && tile.count <= 16) {
    load_y(c0, 0, y);
#pragma unroll 1
    for (; c0 + step < a.D; c0 += step) {
      operand(0, v, o);
      load_w(c0 + step, 0, v);
      load_y(c0 + step, 0, z);
      update(o, 0, y);
      store_y(c0, 0, y);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int h = 0; h < E / S; ++h) y[i][h] = z[i][h];
      }
    }
    if (c0 >= a.D) return;
    operand(0, v, o);
    update(o, 0, y);
    store_y(c0, 0, y);
    return;
  }
#pragma unroll 1
  for (;;) {
    load_y(c0, 0, y);
    operand(0, v, o);
#pragma unroll
    for (int k = 1; k < RB; ++k) {
      __builtin_amdgcn_sched_barrier(0);  // (all at once do not fit the registers)
      load_w(c0, k, v);
      operand(k, v, o);
    }
    int n0 = 0;
#pragma unroll 1
    for (; n0 + 16 < tile.count; n0 += 16) {
      load_y(c0, n0 + 16, z);
      update(o, n0, y);
      store_y(c0, n0, y);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int h = 0; h < E / S; ++h) y[i][h] = z[i][h];
      }
    }
    update(o, n0, y);
    store_y(c0, n0, y);
    c0 += step;
    if (c0 >= a.D) return;
    load_w(c0, 0, v);
  }
}

// ---------------------------------------------------------------- summed over an adapter's tokens

// One workgroup to an adapter, up to 64 ranks and a wave's columns (128, or 64 of fp32
// rows): its waves take blocks of 32 tokens in turn (with those of the other `splits`),
// and their sums are added in order.  A lane loads eight tokens' 16 bytes and
// transposes them; the block's r numbers come straight into the layout of the
// second operand.  The next block's rows are on their way meanwhile.  Both sums of 8,192 tokens
// of 4 adapters by 4,096 columns and 16 ranks: 29.8 us, where reading takes 20; a wave has two
// blocks there, so little of its own overlaps.
constexpr int kOutThreads = 512;
constexpr int kOutWaves = kOutThreads / 64;
template <class TX, int RT>
__global__ void __launch_bounds__(kOutThreads, RT == 1 ? 4 : 2) k_outer(OuterPair pair) {
  const bool second = blockIdx.x >= pair.blocks;
  const OuterArgs& a = pair.a[second];
  const uint32_t block = blockIdx.x - (second ? pair.blocks : 0u);
  constexpr bool BF = TX::BYTES == 2;
  constexpr int E = BF ? 8 : 4;
  constexpr int TERMS = kAdTerms;
  constexpr int C = 16 * E;
  __shared__ float sums[kOutWaves][16][C + 4];
  const int lane = threadIdx.x & 63, m = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // (columns first: workgroups side by side read whole rows)
  const uint32_t item = block / a.chunks;
  const int split = item % a.splits;
  const int g = item / a.splits;
  const int r0 = blockIdx.y * (RT * 16);
  const int64_t c0 = (int64_t)(block % a.chunks) * C;
  const int32_t s = a.start[g], count = a.start[g + 1] - s;
  const int64_t c = c0 + m * E;
  const float scale = a.scales ? a.scales[g] : 1.f;
  f32x4 acc[E][RT];
#pragma unroll
  for (int j = 0; j < E; ++j) {
#pragma unroll
    for (int t = 0; t < RT; ++t) acc[j][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // token of a lane's i-th row: 8 q + i of the block (fp32: 4 i + q).  (No load depends on a
  // condition: past the last token it is that one again, past r or D the last rank and
  // columns.)
  auto at = [&](int i) { return BF ? 8 * q + i : 4 * i + q; };
  const int64_t cx = min(c, (a.D - 1) / E * E) * TX::BYTES;
  int cl[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) cl[t] = min(r0 + 16 * t + m, a.r - 1);
  auto load = [&](int32_t n0, u32x4 (&x)[8], float (&low)[RT][8]) {
    const int32_t mine = a.perm[s + min(n0 + (lane & 31), count - 1)];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t token = __shfl(mine, at(i), 64);
      x[i] = *(const u32x4*)((const char*)a.x + token * a.ldx * TX::BYTES + cx);
#pragma unroll
      for (int t = 0; t < RT; ++t) low[t][i] = a.low.p[token * a.low.ld + cl[t]];
    }
  };
  auto cut = [&](int32_t n0, u32x4 (&x)[8], float (&low)[RT][8]) {
    if (count - n0 >= 32) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool in = n0 + at(i) < count;
#pragma unroll
      for (int d = 0; d < 4; ++d) x[i][d] = in ? x[i][d] : 0u;
#pragma unroll
      for (int t = 0; t < RT; ++t) low[t][i] = in ? low[t][i] : 0.f;
    }
  };
  auto add = [&](const u32x4 (&x)[8], const float (&low)[RT][8]) {
    if constexpr (BF) {
      u32x4 p[RT][TERMS];
#pragma unroll
      for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          uint16_t lo[TERMS], hi[TERMS];
          split_bf16(scale * low[t][i], lo);
          split_bf16(scale * low[t][i + 1], hi);
#pragma unroll
          for (int k = 0; k < TERMS; ++k) p[t][k][i / 2] = lo[k] | (uint32_t)hi[k] << 16;
        }
      }
      // (the 8 by 8 block column by column)
#pragma unroll
      for (int j = 0; j < E; ++j) {
        u32x4 v;
#pragma unroll
        for (int d = 0; d < 4; ++d)
          v[d] = __builtin_amdgcn_perm(x[2 * d + 1][j / 2], x[2 * d][j / 2],
                                       j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
#pragma unroll
          for (int k = TERMS - 1; k >= 0; --k) acc[j][t] = mma_bf16(v, p[t][k], acc[j][t]);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const f32x4 v = __builtin_bit_cast(f32x4, x[i]);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const float f = scale * low[t][i];
#pragma unroll
          for (int j = 0; j < E; ++j) acc[j][t] = mma_f32(v[j], f, acc[j][t]);
        }
      }
    }
  };
  const int32_t step = a.splits * kOutWaves * 32;
  int32_t n0 = (split * kOutWaves + wave) * 32;
  if (n0 < count) {
    u32x4 x[8];
    float low[RT][8];
    load(n0, x, low);
    if constexpr (RT <= 2) {
      u32x4 y[8];
      float lowy[RT][8];
#pragma unroll 1
      for (; (int64_t)n0 + step < count; n0 += step) {
        load(n0 + step, y, lowy);
        add(x, low);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] = y[i];
#pragma unroll
          for (int t = 0; t < RT; ++t) low[t][i] = lowy[t][i];
        }
      }
    } else {  // (both do not fit the registers)
#pragma unroll 1
      for (; (int64_t)n0 + step < count; n0 += step) {
        add(x, low);
        load(n0 + step, x, low);
      }
    }
    cut(n0, x, low);
    add(x, low);
  }
  // lane m holds rank m of each 16, columns (4 q + i) E + j
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    if (t > 0) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int j = 0; j < E; ++j) sums[wave][m][(4 * q + i) * E + j] = acc[j][t][i];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * C / 4; i += kOutThreads) {
      const int rank = r0 + 16 * t + i / (C / 4), at = i % (C / 4) * 4;
      if (rank >= a.r || c0 + at >= a.D) continue;
      float f[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[e] = sums[0][i / (C / 4)][at + e];
#pragma unroll
        for (int v = 1; v < kOutWaves; ++v) f[e] += sums[v][i / (C / 4)][at + e];
      }
      float* out = a.splits == 1
                       ? a.sum + ((int64_t)g * a.r + rank) * a.lds
                       : a.out + (int64_t)split * a.stride + ((int64_t)g * a.r + rank) * a.ldo;
      store_values<InF32, 4>((char*)out, c0 + at, a.D, f);
    }
  }
}

// The parts of t or u, added in order.
__global__ void __launch_bounds__(256) k_low_sum(LowPair pair, int64_t n) {
  const LowArgs& a = pair.a[blockIdx.y];
  if (a.splits <= 1) return;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  float f = a.out[i];
  for (int s = 1; s < a.splits; ++s) f += a.out[(int64_t)s * a.stride + i];
  a.out[i] = f;
}

// The parts of da and db, added in order.
__global__ void __launch_bounds__(256) k_outer_sum(OuterPair pair) {
  const bool second = blockIdx.x >= pair.blocks;
  const OuterArgs& a = pair.a[second];
  const int64_t c = ((int64_t)(blockIdx.x - (second ? pair.blocks : 0u)) * 256 + threadIdx.x) * 4;
  if (c >= a.D || a.splits == 1) return;
  for (int64_t row = blockIdx.y; row < (int64_t)a.G * a.r; row += gridDim.y) {
    const float* p = a.out + row * a.ldo + c;
    f32x4 f = *(const f32x4*)p;
#pragma unroll 4
    for (int s = 1; s < a.splits; ++s) f += *(const f32x4*)(p + s * a.stride);
    const float v[4] = {f[0], f[1], f[2], f[3]};
    store_values<InF32, 4>((char*)(a.sum + row * a.lds), c, a.D, v);
  }
}

template <class TX, class TW, int RT>
hipError_t low_r(const LowPair& p, hipStream_t st) {
  const int64_t tiles = p.a[0].max_tiles;
  const int splits = p.a[0].splits + p.a[1].splits;
  // 32 tokens to a workgroup read the adapter half as often, where that leaves enough of them
  // (4,096 columns, the call: 8,192 tokens of 8 adapters 44.1 us, 44.4 with 16; 2,048 of 4 21.9,
  // 20.6 with 16)
  if constexpr (RT <= 4) {
    if (tiles * splits >= 100) {
      const dim3 grid((unsigned)(tiles * (kAdTile / 32)), (unsigned)splits);
      hipLaunchKernelGGL((k_low<TX, TW, RT, 2>), grid, dim3(kLowThreads), 0, st, p);
      return hipGetLastError();
    }
  }
  const dim3 grid((unsigned)(tiles * (kAdTile / 16)), (unsigned)splits);
  hipLaunchKernelGGL((k_low<TX, TW, RT, 1>), grid, dim3(kLowThreads), 0, st, p);
  return hipGetLastError();
}
template <class TX, class TW>
hipError_t low_t(const LowPair& p, hipStream_t st) {
  const int rt = (p.a[0].r + 15) / 16;
  return rt == 1   ? low_r<TX, TW, 1>(p, st)
         : rt == 2 ? low_r<TX, TW, 2>(p, st)
         : rt <= 4 ? low_r<TX, TW, 4>(p, st)
                   : low_r<TX, TW, 8>(p, st);
}

template <class TW, class TY>
hipError_t expand_t(ExpandArgs a, int64_t N, hipStream_t st) {
  const int64_t span = kExpWaves * 16 * (TW::BYTES == 2 ? 8 : 4);
  const int64_t chunks = (a.D + span - 1) / span;
  // about as many workgroups as stay on the GPU at once; four times as many where tiles are of
  // few tokens, since they differ then, and some have none: the call of 64 tokens of 32 adapters
  // by 151,936 columns 41.3 us (as many 44.4, eight times 44.7), of 8,192 of 8 by 4,096 67.6 (as
  // many 66.7).  Where a tile's workgroups become few, as many are too few: 32,768 of 8 take 241
  // us, and 207 with four times as many.
  int64_t per = (N < 16 * a.max_tiles ? 4096 : 1024) / a.max_tiles;
  a.per = (uint32_t)(per < 1 ? 1 : per < chunks ? per : chunks);
  const dim3 grid((unsigned)(a.max_tiles * a.per));
#define OPD_EXPAND(KL, RB)                                                                \
  if (a.base)                                                                             \
    hipLaunchKernelGGL((k_expand<TW, TY, KL, RB, true>), grid, dim3(kExpThreads), 0, st, a); \
  else                                                                                    \
    hipLaunchKernelGGL((k_expand<TW, TY, KL, RB, false>), grid, dim3(kExpThreads), 0, st, a)
  if (a.r <= 16) {
    OPD_EXPAND(4, 1);
  } else if (a.r <= 32) {
    OPD_EXPAND(8, 1);
  } else if (a.r <= 64) {
    OPD_EXPAND(8, 2);
  } else {
    OPD_EXPAND(8, 4);
  }
#undef OPD_EXPAND
  return hipGetLastError();
}

template <class TX>
hipError_t outer_t(OuterPair p, int count, hipStream_t st) {
  const int64_t span = 16 * (TX::BYTES == 2 ? 8 : 4);
  const int rt = (p.a[0].r + 15) / 16;
  uint32_t blocks[2] = {0, 0};
  for (int i = 0; i < count; ++i) {
    p.a[i].chunks = (uint32_t)((p.a[i].D + span - 1) / span);
    blocks[i] = (uint32_t)(p.a[i].G * p.a[i].splits) * p.a[i].chunks;
  }
  p.blocks = blocks[0];
  const dim3 grid(blocks[0] + blocks[1], (unsigned)(rt <= 4 ? 1 : 2));
  if (rt == 1)
    hipLaunchKernelGGL((k_outer<TX, 1>), grid, dim3(kOutThreads), 0, st, p);
  else if (rt == 2)
    hipLaunchKernelGGL((k_outer<TX, 2>), grid, dim3(kOutThreads), 0, st, p);
  else
    hipLaunchKernelGGL((k_outer<TX, 4>), grid, dim3(kOutThreads), 0, st, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_adapt_plan(const AdaptArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(k_adapt_plan, dim3(1), dim3(kGroupThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_low(const LowPair& p, int x_dt, int w_dt, hipStream_t st) {
  if (w_dt == F32) return low_t<InF32, InF32>(p, st);
  return x_dt == BF16 ? low_t<InBf16, InBf16>(p, st) : low_t<InF32, InBf16>(p, st);
}

hipError_t launch_low_sum(const LowPair& p, int64_t N, hipStream_t st) {
  if (p.a[0].splits <= 1 && p.a[1].splits <= 1) return hipSuccess;
  const int64_t n = N * p.a[0].ldo;
  hipLaunchKernelGGL(k_low_sum, dim3((unsigned)((n + 255) / 256), p.a[1].splits > 0 ? 2 : 1),
                     dim3(256), 0, st, p, n);
  return hipGetLastError();
}

hipError_t launch_expand(const ExpandArgs& a, int64_t N, int w_dt, int y_dt, hipStream_t st) {
  if (w_dt == F32) return expand_t<InF32, InF32>(a, N, st);
  return y_dt == BF16 ? expand_t<InBf16, InBf16>(a, N, st) : expand_t<InBf16, InF32>(a, N, st);
}

hipError_t launch_outer(const OuterPair& pair, int x_dt, int y_dt, hipStream_t st) {
  hipError_t e;
  if (x_dt == y_dt) {
    e = x_dt == BF16 ? outer_t<InBf16>(pair, 2, st) : outer_t<InF32>(pair, 2, st);
  } else {  // bf16 x, fp32 dy
    OuterPair one = pair;
    e = outer_t<InBf16>(one, 1, st);
    if (e != hipSuccess) return e;
    one.a[0] = pair.a[1];
    e = outer_t<InF32>(one, 1, st);
  }
  if (e != hipSuccess || (pair.a[0].splits == 1 && pair.a[1].splits == 1)) return e;
  OuterPair p = pair;
  const int64_t rows = (int64_t)p.a[0].G * p.a[0].r;
  const int64_t x = (p.a[0].D + 1023) / 1024, y = (p.a[1].D + 1023) / 1024;
  p.blocks = (uint32_t)x;
  hipLaunchKernelGGL(k_outer_sum, dim3((unsigned)(x + y), (unsigned)(rows < 65535 ? rows : 65535)),
                     dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace opd
