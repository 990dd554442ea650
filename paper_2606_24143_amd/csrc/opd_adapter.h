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
// Sums are fp32; t and u pass to the second product as two bf16 parts for bf16 results
// (2^-17 of them), three for fp32 ones (2^-25).  fp32 operands take the fp32
// matrix instructions, exact products throughout.
#pragma once

#include "opd_device.h"
#include "opd_group.h"
#include "opd_model.h"

namespace opd {
namespace {

typedef __bf16 BFrag __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------- tokens by adapter

struct PlanLds {
  GroupLds group;
  uint32_t tile[kGroupKeys + 1];
};

// One workgroup: tokens sorted by adapter (key G: none, G + 1: an id outside [0, G)),
// and tiles of kAdTile tokens of one key.
__global__ void __launch_bounds__(kGroupThreads) k_adapt_plan(AdaptArgs a) {
  __shared__ PlanLds sh;
  const int32_t G = a.G;
  const int32_t* ids = a.ids;
  const int count = G + 2;
  uint32_t end;
  const uint32_t first = group_tokens(
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
    a.start[threadIdx.x] = (int32_t)first;
  }
  if ((int)threadIdx.x == count) {
    place[count] = end;
    a.start[count] = (int32_t)end;
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

// ---------------------------------------------------------------- loads

template <class T>
using Elem = std::conditional_t<T::BYTES == 2, uint16_t, uint32_t>;

// Eight (bf16) or four (fp32) consecutive elements of a row, 16 bytes; those at or
// past `end` are 0.
template <class T>
__device__ __forceinline__ u32x4 load16(const char* row, int64_t c, int64_t end) {
  constexpr int E = 16 / T::BYTES;
  if (c + E <= end) return *(const u32x4*)(row + c * T::BYTES);
  u32x4 r = {0, 0, 0, 0};
  if (c < end) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (c + e >= end) continue;
      const uint32_t b = ((const Elem<T>*)row)[c + e];
      if constexpr (T::BYTES == 2)
        r[e / 2] |= b << (16 * (e & 1));
      else
        r[e] = b;
    }
  }
  return r;
}
// Four consecutive elements widened to fp32.
template <class T>
__device__ __forceinline__ f32x4 load4_wide(const char* row, int64_t c, int64_t end) {
  f32x4 f = {0.f, 0.f, 0.f, 0.f};
  if (c + 4 <= end) {
    if constexpr (T::BYTES == 2) {
      const u32x2 x = *(const u32x2*)(row + c * 2);
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        f[2 * d] = __uint_as_float(x[d] << 16);
        f[2 * d + 1] = __uint_as_float(x[d] & 0xFFFF0000u);
      }
    } else {
      f = *(const f32x4*)(row + c * 4);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < end) f[e] = load_elem<T>(row, c + e);
  }
  return f;
}

// In: row t of an 8 by 8 block of bf16 (16 bytes).  Out: column j, of all eight rows.
__device__ __forceinline__ void transpose8(const u32x4 (&in)[8], u32x4 (&out)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const uint32_t lo = in[2 * d][j / 2], hi = in[2 * d + 1][j / 2];
      out[j][d] = __builtin_amdgcn_perm(hi, lo, j & 1 ? 0x07060302u : 0x05040100u);
    }
  }
}

__device__ __forceinline__ f32x4 mma_bf16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(BFrag, a),
                                                 __builtin_bit_cast(BFrag, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma_f32(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// A number as TERMS bf16 parts that add up to it (to 2^-9, 2^-17, 2^-25 of it); one that
// is not finite in bf16 is its first part.
template <int TERMS>
__device__ __forceinline__ void split_bf16(float f, uint16_t (&p)[TERMS]) {
#pragma unroll
  for (int i = 0; i < TERMS; ++i) {
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

// One workgroup to 16 tokens of an adapter and a part of the long axis: its waves
// take steps of 64 (bf16) or 32 (fp32) columns in turn, and their sums are added in
// order.  RT: ranks / 16.
constexpr int kLowThreads = 512;
constexpr int kLowWaves = kLowThreads / 64;
template <class TX, class TW, int RT>
__global__ void __launch_bounds__(kLowThreads) k_low(LowArgs a) {
  constexpr bool BF = TX::BYTES == 2 && TW::BYTES == 2;
  constexpr int STEP = BF ? 64 : 32;
  __shared__ float sums[kLowWaves][16][RT * 16 + 1];
  const int sub = blockIdx.x % (kAdTile / 16);
  const AdTile tile = a.tiles[blockIdx.x / (kAdTile / 16)];
  if (sub * 16 >= tile.count || tile.key >= a.G) return;
  const int lane = threadIdx.x & 63, m = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int count = min(16, tile.count - sub * 16);
  const int32_t* perm = a.perm + tile.pos + sub * 16;
  const char* x = (const char*)a.x + (int64_t)perm[min(m, count - 1)] * a.ldx * TX::BYTES;
  const char* w = (const char*)a.w + ((int64_t)tile.key * a.r + m) * a.ldw * TW::BYTES;
  f32x4 acc[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int64_t d0 = (int64_t)blockIdx.y * a.span;
  const int64_t d1 = d0 + a.span < a.D ? d0 + a.span : a.D;
  for (int64_t d = d0 + wave * STEP; d < d1; d += kLowWaves * STEP) {
    if constexpr (BF) {
      // (columns d + 16 q .. + 16 of both, 32 bytes a lane: two instructions' worth)
      const int64_t c = d + 16 * q;
      u32x4 xv[2], wv[RT][2];
#pragma unroll
      for (int i = 0; i < 2; ++i) xv[i] = load16<TX>(x, c + 8 * i, d1);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          wv[t][i] = u32x4{0, 0, 0, 0};
          if (16 * t + m < a.r)
            wv[t][i] = load16<TW>(w + (int64_t)t * 16 * a.ldw * TW::BYTES, c + 8 * i, d1);
        }
      }
#pragma unroll
      for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int i = 0; i < 2; ++i) acc[t] = mma_bf16(xv[i], wv[t][i], acc[t]);
      }
    } else {
      const int64_t c = d + 8 * q;
      f32x4 xv[2], wv[RT][2];
#pragma unroll
      for (int i = 0; i < 2; ++i) xv[i] = load4_wide<TX>(x, c + 4 * i, d1);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          wv[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
          if (16 * t + m < a.r)
            wv[t][i] = load4_wide<TW>(w + (int64_t)t * 16 * a.ldw * TW::BYTES, c + 4 * i, d1);
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
          for (int t = 0; t < RT; ++t) acc[t] = mma_f32(xv[i][e], wv[t][i][e], acc[t]);
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) {
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[wave][4 * q + i][16 * t + m] = acc[t][i];
  }
  __syncthreads();
  float* out = a.out + (int64_t)blockIdx.y * a.stride;
  for (int i = threadIdx.x; i < count * a.r; i += kLowThreads) {
    const int n = i / a.r, c = i % a.r;
    float f = sums[0][n][c];
#pragma unroll
    for (int v = 1; v < kLowWaves; ++v) f += sums[v][n][c];
    out[(int64_t)perm[n] * a.ldo + c] = f;
  }
}

// ---------------------------------------------------------------- the r numbers times the rows

// Columns of a wave's tile: lane m = 4 i + j of an operand has the columns of piece
// 4 j + i, so that the four lanes that hold a token's results hold consecutive pieces.
__device__ __forceinline__ int piece(int m) { return (m & 3) * 4 + (m >> 2); }

constexpr int kExpThreads = 256;
constexpr int kExpWaves = kExpThreads / 64;

// E values of a row of the result, and back.
template <class T, int E>
__device__ __forceinline__ void load_values(const char* row, int64_t c, int64_t end, float (&f)[E]) {
#pragma unroll
  for (int v = 0; v < E / 4; ++v) {
    const f32x4 x = load4_wide<T>(row, c + 4 * v, end);
#pragma unroll
    for (int e = 0; e < 4; ++e) f[4 * v + e] = x[e];
  }
}
template <class T, int E>
__device__ __forceinline__ void store_values(char* row, int64_t c, int64_t end, const float (&f)[E]) {
  if (c + E <= end) {
    if constexpr (T::BYTES == 2) {
      if constexpr (E == 8)
        *(u32x4*)(row + c * 2) = u32x4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]),
                                       pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
      else
        *(u32x2*)(row + c * 2) = u32x2{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])};
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

// One workgroup to a tile of up to kAdTile tokens of an adapter and 4 waves' columns
// (128 each, or 64 of fp32 rows): a wave keeps its columns of the adapter in
// registers and passes over the tokens, 16 at a time.  The shared projection's values
// are what the sums start from.  RB: ranks / 32.
template <class TW, class TY, int RB>
__global__ void __launch_bounds__(kExpThreads) k_expand(ExpandArgs a) {
  constexpr bool BF = TW::BYTES == 2;
  constexpr int E = BF ? 8 : 4;          // columns of a piece
  constexpr int TERMS = TY::BYTES == 2 ? 2 : 3;
  constexpr int KP = BF ? RB * 32 + 8 : RB * 32 + 4;  // (padded: lanes of a read spread over the banks)
  __shared__ __align__(16) uint16_t part[BF ? TERMS : 1][BF ? kAdTile : 1][KP];
  __shared__ float wide[BF ? 1 : kAdTile][BF ? 1 : KP];
  const AdTile tile = a.tiles[blockIdx.x];
  if (tile.count == 0) return;
  const int lane = threadIdx.x & 63, m = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t* perm = a.perm + tile.pos;
  const int64_t c0 = ((int64_t)blockIdx.y * kExpWaves + wave) * (16 * E);
  const bool live = tile.key < a.G;
  if (!live && tile.key == a.G && a.base == a.out) return;  // in place: as it is
  // this wave's columns of the adapter, ranks along a lane
  u32x4 wb[BF ? RB : 1][8];
  f32x4 wf[BF ? 1 : RB * 8];
  if (live) {
    const char* w = (const char*)a.w + (int64_t)tile.key * a.r * a.ldw * TW::BYTES;
    const int64_t c = c0 + piece(m) * E;
    if constexpr (BF) {
#pragma unroll
      for (int k = 0; k < RB; ++k) {
        u32x4 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int rank = 32 * k + 8 * q + i;
          v[i] = u32x4{0, 0, 0, 0};
          if (rank < a.r) v[i] = load16<TW>(w + (int64_t)rank * a.ldw * 2, c, a.D);
        }
        transpose8(v, wb[k]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < RB * 8; ++k) {
        const int rank = 4 * k + q;
        wf[k] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (rank < a.r) wf[k] = load4_wide<TW>(w + (int64_t)rank * a.ldw * 4, c, a.D);
      }
    }
    const float scale = a.scales ? a.scales[tile.key] : 1.f;
    for (int i = threadIdx.x; i < kAdTile * RB * 32; i += kExpThreads) {
      const int n = i / (RB * 32), k = i % (RB * 32);
      float f = 0.f;
      if (n < tile.count) {
        f = low_value(a.low, perm[n], k);
        if (a.low_out && blockIdx.y == 0 && k < a.r) a.low_out[(int64_t)perm[n] * a.r + k] = f;
        f *= scale;
      }
      if constexpr (BF) {
        uint16_t p[TERMS];
        split_bf16<TERMS>(f, p);
#pragma unroll
        for (int t = 0; t < TERMS; ++t) part[t][n][k] = p[t];
      } else {
        wide[n][k] = f;
      }
    }
  } else if (a.low_out && blockIdx.y == 0) {
    for (int i = threadIdx.x; i < tile.count * a.r; i += kExpThreads)
      a.low_out[(int64_t)perm[i / a.r] * a.r + i % a.r] =
          tile.key == a.G ? 0.f : __builtin_nanf("");
  }
  __syncthreads();
#pragma unroll 1
  for (int n0 = 0; n0 < tile.count; n0 += 16) {
    const bool mine = n0 + m < tile.count;
    const int64_t token = perm[mine ? n0 + m : tile.count - 1];
    // pieces 4 i + q of the wave's columns
    float y[4][E];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int e = 0; e < E; ++e) y[i][e] = tile.key == a.G + 1 ? __builtin_nanf("") : 0.f;
      const int64_t c = c0 + (4 * i + q) * E;
      if (a.base && tile.key <= a.G && c < a.D)
        load_values<TY, E>((const char*)a.base + token * a.ldb * TY::BYTES, c, a.D, y[i]);
    }
    if (live) {
#pragma unroll
      for (int j = 0; j < E; ++j) {
        f32x4 acc = {y[0][j], y[1][j], y[2][j], y[3][j]};
        if constexpr (BF) {
#pragma unroll
          for (int k = 0; k < RB; ++k) {
#pragma unroll
            for (int t = TERMS - 1; t >= 0; --t)
              acc = mma_bf16(wb[k][j], *(const u32x4*)&part[t][n0 + m][32 * k + 8 * q], acc);
          }
        } else {
#pragma unroll
          for (int k = 0; k < RB * 8; ++k) acc = mma_f32(wf[k][j], wide[n0 + m][4 * k + q], acc);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i][j] = acc[i];
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t c = c0 + (4 * i + q) * E;
      if (mine && c < a.D)
        store_values<TY, E>((char*)a.out + token * a.ldo * TY::BYTES, c, a.D, y[i]);
    }
  }
}

// ---------------------------------------------------------------- summed over an adapter's tokens

// One workgroup to an adapter, up to 64 ranks, 4 waves' columns, and every `splits`-th
// block of 32 tokens.  A lane loads eight tokens' 16 bytes and transposes them.
constexpr int kOutThreads = 256;
constexpr int kOutWaves = kOutThreads / 64;
template <class TX, int RT>
__global__ void __launch_bounds__(kOutThreads) k_outer(OuterArgs a) {
  constexpr bool BF = TX::BYTES == 2;
  constexpr int E = BF ? 8 : 4;
  constexpr int TERMS = 3;
  constexpr int KP = BF ? 32 + 8 : 32 + 1;
  __shared__ __align__(16) uint16_t part[BF ? TERMS : 1][BF ? RT * 16 : 1][KP];
  __shared__ float wide[BF ? 1 : RT * 16][BF ? 1 : KP];
  const int lane = threadIdx.x & 63, m = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = blockIdx.x % a.splits;
  const int g = blockIdx.x / a.splits;
  const int r0 = blockIdx.z * (RT * 16);
  const int64_t c0 = ((int64_t)blockIdx.y * kOutWaves + wave) * (16 * E);
  const int32_t s = a.start[g], count = a.start[g + 1] - s;
  const int64_t c = c0 + piece(m) * E;
  const float scale = a.scales ? a.scales[g] : 1.f;
  f32x4 acc[E][RT];
#pragma unroll
  for (int j = 0; j < E; ++j) {
#pragma unroll
    for (int t = 0; t < RT; ++t) acc[j][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
#pragma unroll 1
  for (int32_t n0 = split * 32; n0 < count; n0 += a.splits * 32) {
    const int32_t* perm = a.perm + s + n0;
    const int here = min(32, count - n0);
    __syncthreads();
    for (int i = threadIdx.x; i < RT * 16 * 32; i += kOutThreads) {
      const int n = i / (RT * 16), k = i % (RT * 16);
      const float f = n < here ? scale * low_value(a.low, perm[n], r0 + k) : 0.f;
      if constexpr (BF) {
        uint16_t p[TERMS];
        split_bf16<TERMS>(f, p);
#pragma unroll
        for (int t = 0; t < TERMS; ++t) part[t][k][n] = p[t];
      } else {
        wide[k][n] = f;
      }
    }
    __syncthreads();
    if constexpr (BF) {
      u32x4 x[8], v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int n = 8 * q + i;
        x[i] = u32x4{0, 0, 0, 0};
        if (n < here) x[i] = load16<TX>((const char*)a.x + (int64_t)perm[n] * a.ldx * 2, c, a.D);
      }
      transpose8(x, v);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int p = TERMS - 1; p >= 0; --p) {
          const u32x4 low = *(const u32x4*)&part[p][16 * t + m][8 * q];
#pragma unroll
          for (int j = 0; j < E; ++j) acc[j][t] = mma_bf16(v[j], low, acc[j][t]);
        }
      }
    } else {
      f32x4 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int n = 4 * i + q;
        x[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (n < here) x[i] = load4_wide<TX>((const char*)a.x + (int64_t)perm[n] * a.ldx * 4, c, a.D);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const float low = wide[16 * t + m][4 * i + q];
#pragma unroll
          for (int j = 0; j < E; ++j) acc[j][t] = mma_f32(x[i][j], low, acc[j][t]);
        }
      }
    }
  }
  // lane m holds rank m of each 16, piece 4 i + q of the columns
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int rank = r0 + 16 * t + m;
    if (rank >= a.r) continue;
    float* out = a.out + (int64_t)split * a.stride + ((int64_t)g * a.r + rank) * a.ldo;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t at = c0 + (4 * i + q) * E;
      if (at >= a.D) continue;
      float f[E];
#pragma unroll
      for (int j = 0; j < E; ++j) f[j] = acc[j][t][i];
      store_values<InF32, E>((char*)out, at, a.D, f);
    }
  }
}

// The parts of da or db, added in order.
__global__ void __launch_bounds__(256) k_outer_sum(OuterArgs a, float* out, int64_t ldo) {
  const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (c >= a.D) return;
  for (int64_t row = blockIdx.y; row < (int64_t)a.G * a.r; row += gridDim.y) {
    const float* p = a.out + row * a.ldo + c;
    f32x4 f = *(const f32x4*)p;
    for (int s = 1; s < a.splits; ++s) f += *(const f32x4*)(p + s * a.stride);
    const float v[4] = {f[0], f[1], f[2], f[3]};
    store_values<InF32, 4>((char*)(out + row * ldo), c, a.D, v);
  }
}

template <class TX, class TW>
hipError_t low_t(const LowArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.max_tiles * (kAdTile / 16)), (unsigned)a.splits);
  const int rt = (a.r + 15) / 16;
  if (rt == 1)
    hipLaunchKernelGGL((k_low<TX, TW, 1>), grid, dim3(kLowThreads), 0, st, a);
  else if (rt == 2)
    hipLaunchKernelGGL((k_low<TX, TW, 2>), grid, dim3(kLowThreads), 0, st, a);
  else if (rt <= 4)
    hipLaunchKernelGGL((k_low<TX, TW, 4>), grid, dim3(kLowThreads), 0, st, a);
  else
    hipLaunchKernelGGL((k_low<TX, TW, 8>), grid, dim3(kLowThreads), 0, st, a);
  return hipGetLastError();
}

template <class TW, class TY>
hipError_t expand_t(const ExpandArgs& a, hipStream_t st) {
  const int64_t span = kExpWaves * 16 * (TW::BYTES == 2 ? 8 : 4);
  const dim3 grid((unsigned)a.max_tiles, (unsigned)((a.D + span - 1) / span));
  const int rb = (a.r + 31) / 32;
  if (rb == 1)
    hipLaunchKernelGGL((k_expand<TW, TY, 1>), grid, dim3(kExpThreads), 0, st, a);
  else if (rb == 2)
    hipLaunchKernelGGL((k_expand<TW, TY, 2>), grid, dim3(kExpThreads), 0, st, a);
  else
    hipLaunchKernelGGL((k_expand<TW, TY, 4>), grid, dim3(kExpThreads), 0, st, a);
  return hipGetLastError();
}

template <class TX>
hipError_t outer_t(const OuterArgs& a, hipStream_t st) {
  const int64_t span = kOutWaves * 16 * (TX::BYTES == 2 ? 8 : 4);
  const int rt = (a.r + 15) / 16;
  const dim3 grid((unsigned)(a.G * a.splits), (unsigned)((a.D + span - 1) / span),
                  (unsigned)(rt <= 4 ? 1 : 2));
  if (rt == 1)
    hipLaunchKernelGGL((k_outer<TX, 1>), grid, dim3(kOutThreads), 0, st, a);
  else if (rt == 2)
    hipLaunchKernelGGL((k_outer<TX, 2>), grid, dim3(kOutThreads), 0, st, a);
  else
    hipLaunchKernelGGL((k_outer<TX, 4>), grid, dim3(kOutThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_adapt_plan(const AdaptArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(k_adapt_plan, dim3(1), dim3(kGroupThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_low(const LowArgs& a, int x_dt, int w_dt, hipStream_t st) {
  if (w_dt == F32) return low_t<InF32, InF32>(a, st);
  return x_dt == BF16 ? low_t<InBf16, InBf16>(a, st) : low_t<InF32, InBf16>(a, st);
}

hipError_t launch_expand(const ExpandArgs& a, int w_dt, int y_dt, hipStream_t st) {
  if (w_dt == F32) return expand_t<InF32, InF32>(a, st);
  return y_dt == BF16 ? expand_t<InBf16, InBf16>(a, st) : expand_t<InBf16, InF32>(a, st);
}

hipError_t launch_outer(const OuterArgs& a, int x_dt, float* out, int64_t ldo, hipStream_t st) {
  OuterArgs b = a;
  if (a.splits == 1) {
    b.out = out;
    b.ldo = ldo;
  }
  const hipError_t e = x_dt == BF16 ? outer_t<InBf16>(b, st) : outer_t<InF32>(b, st);
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t rows = (int64_t)a.G * a.r;
  hipLaunchKernelGGL(k_outer_sum, dim3((unsigned)((a.D + 1023) / 1024), (unsigned)(rows < 65535 ? rows : 65535)),
                     dim3(256), 0, st, b, out, ldo);
  return hipGetLastError();
}

}  // namespace opd
