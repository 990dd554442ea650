// Token embeddings: rows of a vocabulary-sized table by token, and the table's
// gradient (the learner's update reaches the table, which is often the output
// head's too).
//   lookup    out[n, :] = scale * table[ids[n], :]
//   gradient  dtable[v, :] = scale * sum over tokens n of id v of dy[n, :]
// Id -1 (what the calls that roll out write past a sequence's last token) is a row
// of zeros and adds to nothing; any other id outside [0, V) a row of NaN.
// Both are bound by HBM: the lookup reads and writes each element once, the
// gradient writes a table that is mostly zeros.
#pragma once

#include "opd_device.h"
#include "opd_group.h"
#include "opd_model.h"

namespace opd {
namespace {

constexpr int kEmbThreads = 256;
constexpr int kEmbWaves = kEmbThreads / 64;

// E consecutive elements of a row, widened.
template <class TI, int E>
__device__ __forceinline__ void load_wide(const char* row, int64_t c, int64_t H, float (&f)[E]) {
  if (c + E <= H) {
    if constexpr (TI::BYTES == 2) {
      if constexpr (E == 8) {
        const u32x4 x = *(const u32x4*)(row + c * 2);
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          f[2 * d] = __uint_as_float(x[d] << 16);
          f[2 * d + 1] = __uint_as_float(x[d] & 0xFFFF0000u);
        }
      } else {
        const u32x2 x = *(const u32x2*)(row + c * 2);
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          f[2 * d] = __uint_as_float(x[d] << 16);
          f[2 * d + 1] = __uint_as_float(x[d] & 0xFFFF0000u);
        }
      }
    } else {
#pragma unroll
      for (int v = 0; v < E / 4; ++v) {
        const f32x4 x = *(const f32x4*)(row + c * 4 + 16 * v);
#pragma unroll
        for (int d = 0; d < 4; ++d) f[4 * v + d] = x[d];
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = c + e < H ? load_elem<TI>(row, c + e) : 0.f;
  }
}

// The same back, rounded to the row's type (columns past H are not written).
template <class TO, int E, bool NT>
__device__ __forceinline__ void store_wide(char* row, int64_t c, int64_t H, const float (&f)[E]) {
  if (c + E <= H) {
    if constexpr (TO::BYTES == 2) {
      if constexpr (E == 8) {
        const u32x4 x = {pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]),
                         pack_bf16x2(f[6], f[7])};
        if constexpr (NT)
          __builtin_nontemporal_store(x, (u32x4*)(row + c * 2));
        else
          *(u32x4*)(row + c * 2) = x;
      } else {
        const u32x2 x = {pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])};
        if constexpr (NT)
          __builtin_nontemporal_store(x, (u32x2*)(row + c * 2));
        else
          *(u32x2*)(row + c * 2) = x;
      }
    } else {
#pragma unroll
      for (int v = 0; v < E / 4; ++v) {
        const f32x4 x = {f[4 * v], f[4 * v + 1], f[4 * v + 2], f[4 * v + 3]};
        if constexpr (NT)
          __builtin_nontemporal_store(x, (f32x4*)(row + c * 4 + 16 * v));
        else
          *(f32x4*)(row + c * 4 + 16 * v) = x;
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (c + e >= H) continue;
      if constexpr (TO::BYTES == 2)
        ((__bf16*)row)[c + e] = (__bf16)f[e];
      else
        ((float*)row)[c + e] = f[e];
    }
  }
}

// ---------------------------------------------------------------- lookup

// One wavefront to a token and a chunk of 64 * E * VPL columns, four to a
// workgroup.  E: elements of a lane's store (16 bytes of it).  32,768 tokens of 8 KiB, some
// frequent: 80 us, 75 at a copy's rate; with one vector to a lane 91.
template <class TI, class TO, int VPL>
__global__ void __launch_bounds__(kEmbThreads) k_embed(EmbedArgs a) {
  constexpr int E = 16 / TO::BYTES;
  const uint32_t u = blockIdx.x * kEmbWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (u >= a.units) return;
  const int64_t n = a.row0 + u / a.chunks;
  const int64_t c0 = (int64_t)(u % a.chunks) * (64 * E * VPL) + (threadIdx.x & 63) * E;
  const int32_t id = a.ids[n];
  char* out = (char*)a.out + n * a.ldo * TO::BYTES;
  float f[VPL][E];
  if (id >= 0 && id < a.V) {
    const char* row = (const char*)a.table + (int64_t)id * a.ld * TI::BYTES;
#pragma unroll
    for (int v = 0; v < VPL; ++v)
      if (c0 + v * 64 * E < a.H) load_wide<TI, E>(row, c0 + v * 64 * E, a.H, f[v]);
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
#pragma unroll
      for (int e = 0; e < E; ++e) f[v][e] *= a.scale;
    }
  } else {
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
#pragma unroll
      for (int e = 0; e < E; ++e) f[v][e] = id == -1 ? 0.f : __builtin_nanf("");
    }
  }
#pragma unroll
  for (int v = 0; v < VPL; ++v)
    if (c0 + v * 64 * E < a.H) store_wide<TO, E, false>(out, c0 + v * 64 * E, a.H, f[v]);
}

// ---------------------------------------------------------------- gradient

// Tokens sorted by id: start[v] the first place of entry v, perm the tokens.  16,384 tokens and
// 151,936 entries: 19 us, two passes over all ids by each workgroup.
__global__ void __launch_bounds__(kGroupThreads) k_embed_group(EmbedGradArgs a) {
  __shared__ GroupLds<kEmbKeys> sh;
  const int32_t lo = (int32_t)((int64_t)blockIdx.x * a.keys);
  const int count = (int)(a.V - lo < a.keys ? a.V - lo : a.keys);
  const int32_t* ids = a.ids;
  const int64_t V = a.V;
  uint32_t end;
  const uint32_t first = group_tokens<kEmbKeys, true>(
      a.N, lo, count, [=](int64_t n) { return (uint32_t)ids[n] < (uint32_t)V ? ids[n] : -1; },
      a.perm, sh, end);
  if ((int)threadIdx.x < count) a.start[lo + (int)threadIdx.x] = (int32_t)first;
  if (threadIdx.x == 0 && lo + count == a.V) a.start[a.V] = (int32_t)end;
}

// Adds dy[token, c + 256 v ..] for the tokens that lanes [0, count) hold, in order; B rows on
// their way at once.  (Every lane takes part, since every lane's token is read: those whose
// columns lie past H load nothing.)
template <class TI, int VPL, int B>
__device__ __forceinline__ void add_rows(const EmbedGradArgs& a, int32_t token, int count,
                                         int64_t c, float (&f)[VPL][4]) {
#pragma unroll 1
  for (int i = 0; i < count; i += B) {
    float x[B][VPL][4];
#pragma unroll
    for (int b = 0; b < B; ++b) {
      if (i + b >= count) continue;
      const char* row =
          (const char*)a.dy + (int64_t)__builtin_amdgcn_readlane(token, i + b) * a.ldy * TI::BYTES;
#pragma unroll
      for (int v = 0; v < VPL; ++v) load_wide<TI, 4>(row, c + 256 * v, a.H, x[b][v]);
    }
#pragma unroll
    for (int b = 0; b < B; ++b) {
      if (i + b >= count) continue;
#pragma unroll
      for (int v = 0; v < VPL; ++v) {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[v][e] += x[b][v][e];
      }
    }
  }
}

template <class TO, int E>
__device__ __forceinline__ void store_sum(const EmbedGradArgs& a, int64_t v, int64_t c,
                                          float (&f)[E]) {
  char* row = (char*)a.out + v * a.ldo * TO::BYTES;
#pragma unroll
  for (int e = 0; e < E; ++e) f[e] *= a.scale;
  if (a.accumulate) {
    float x[E];
    load_wide<TO, E>(row, c, a.H, x);
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] += x[e];
  }
  store_wide<TO, E, true>(row, c, a.H, f);
}

// Two launches: the entries with tokens are read and summed, then the empty ones are filled
// (most of the table, as a rule).  A wavefront that waits for a row holds a place among the
// stores: in one launch 16,384 tokens of 8 KiB cost 200 us beside the fill's 350, apart
// they cost 73.
//
// Entries of more than kEmbTile tokens are summed tile by tile of the sorted tokens, so
// that one frequent token does not keep one wavefront busy, and the tiles' sums are added
// in the second launch.  A tile holds a part of at most two such entries: one that begins
// before or at its first place (part 0), and one that begins inside it (part 1) and goes
// on past it.

// A tile's long entries, by a wavefront whose lanes hold the tile's tokens.
struct TileLane {
  int32_t token, id, s, e;  // the lane's token, its entry, and that one's places
  bool many;
};
__device__ __forceinline__ TileLane tile_lane(const EmbedGradArgs& a, int64_t tile) {
  const int lane = threadIdx.x & 63;
  const int64_t p = tile * kEmbTile + lane, kept = a.start[a.V];
  TileLane t = {0, -1, 0, 0, false};
  if (lane < kEmbTile && p < kept) {
    t.token = a.perm[p];
    t.id = a.ids[t.token];
    t.s = a.start[t.id];
    t.e = a.start[t.id + 1];
    t.many = t.e - t.s > kEmbTile;
  }
  return t;
}

// One wavefront to a tile, or to the entry whose tokens begin at a place of the sorted ones,
// and a chunk of 256 VPL columns.  (Bound by the chains of dependent loads: a place's token,
// its entry, the entry's places, its rows.  16,384 tokens of 8 KiB: 512 columns and 4 rows
// at once 73 us, 512 and 8 95, 1,024 and 4 105, 256 and 8 88: more registers, fewer waves.)
template <class TI, class TO, int VPL>
__global__ void __launch_bounds__(kEmbThreads) k_embed_sums(EmbedGradArgs a) {
  const uint32_t u = blockIdx.x * kEmbWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (u >= a.units) return;
  const int lane = threadIdx.x & 63;
  const int64_t row = a.row0 + u / a.chunks;
  const int64_t c = (int64_t)(u % a.chunks) * (256 * VPL) + lane * 4;
  float f[VPL][4] = {};
  if (row < a.tiles) {
    const TileLane t = tile_lane(a, row);
#pragma unroll 1
    for (int part = 0; part < 2; ++part) {
      const uint64_t in = __ballot(t.many && (part == 0) == (t.s <= row * kEmbTile));
      if (!in) continue;
      // (its places are consecutive: moved down to lane 0)
      const int first = __ffsll((long long)in) - 1, count = __popcll(in);
      const int32_t mine = __shfl(t.token, (first + lane) & 63, 64);
#pragma unroll
      for (int v = 0; v < VPL; ++v) {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[v][e] = 0.f;
      }
      add_rows<TI, VPL, 8 / VPL>(a, mine, count, c, f);
      float* to = a.partial + (row * 2 + part) * a.hp + c;
#pragma unroll
      for (int v = 0; v < VPL; ++v)
        if (c + 256 * v < a.H) *(f32x4*)(to + 256 * v) = f32x4{f[v][0], f[v][1], f[v][2], f[v][3]};
    }
    return;
  }
  const int64_t p = row - a.tiles;
  if (p >= a.start[a.V]) return;
  const int32_t v = a.ids[a.perm[p]];
  const int32_t s = a.start[v], e = a.start[v + 1];
  if (s != p || e - s > kEmbTile) return;
  add_rows<TI, VPL, 8 / VPL>(a, lane < e - s ? a.perm[s + lane] : 0, e - s, c, f);
#pragma unroll
  for (int i = 0; i < VPL; ++i)
    if (c + 256 * i < a.H) store_sum<TO, 4>(a, v, c + 256 * i, f[i]);
}

// One wavefront to a tile, or an entry, and a chunk of 64 E columns, a store of 16 bytes to a
// lane: the tiles' sums of a long entry, in order, by the wavefronts of the tile that it
// begins in; and zeros where there is no token.  (One store to a lane, in short waves
// side by side, is as fast as a plain fill: 370 us where one takes 361, for 151,936 by 4,096
// fp32.  Four stores to a lane took 425, eight rows to a wave 440.)
template <class TO>
__global__ void __launch_bounds__(kEmbThreads) k_embed_rest(EmbedGradArgs a) {
  constexpr int E = 16 / TO::BYTES;
  const uint32_t u = blockIdx.x * kEmbWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (u >= a.units) return;
  const int lane = threadIdx.x & 63;
  const int64_t row = a.row0 + u / a.chunks;
  const int64_t c = (int64_t)(u % a.chunks) * (64 * E) + lane * E;
  float f[E] = {};
  int64_t v = row - a.tiles;
  if (v >= 0) {
    if (a.start[v] != a.start[v + 1]) return;
    if (c < a.H) store_wide<TO, E, true>((char*)a.out + v * a.ldo * TO::BYTES, c, a.H, f);
    return;
  }
  const TileLane t = tile_lane(a, row);
  // (at most one begins here: it goes on past the tile)
  const uint64_t in = __ballot(t.many && t.s == row * kEmbTile + lane);
  if (!in) return;
  const int l = __ffsll((long long)in) - 1;
  v = __builtin_amdgcn_readlane(t.id, l);
  const int64_t s = __builtin_amdgcn_readlane(t.s, l), e = __builtin_amdgcn_readlane(t.e, l);
  if (c >= a.H) return;
  const int64_t t1 = (e + kEmbTile - 1) / kEmbTile;
  f32x4 sum[E / 4];
  const float* from = a.partial + (row * 2 + (s > row * kEmbTile ? 1 : 0)) * a.hp + c;
#pragma unroll
  for (int k = 0; k < E / 4; ++k) sum[k] = *(const f32x4*)(from + 4 * k);
#pragma unroll 8
  for (int64_t i = row + 1; i < t1; ++i) {
#pragma unroll
    for (int k = 0; k < E / 4; ++k) sum[k] += *(const f32x4*)(a.partial + i * 2 * a.hp + c + 4 * k);
  }
#pragma unroll
  for (int k = 0; k < E; ++k) f[k] = sum[k / 4][k % 4];
  store_sum<TO, E>(a, v, c, f);
}

// Few tokens, in one launch: a wavefront looks for its entry's tokens among the ids itself.
template <class TI, class TO>
__global__ void __launch_bounds__(kEmbThreads) k_embed_few(EmbedGradArgs a) {
  const uint32_t u = blockIdx.x * kEmbWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (u >= a.units) return;
  const int lane = threadIdx.x & 63;
  const int64_t v = a.row0 + u / a.chunks;
  const int64_t c = (int64_t)(u % a.chunks) * 256 + lane * 4;
  float f[1][4] = {};
  bool any = false;
  for (int64_t n = 0; n < a.N; n += 64) {
    const int32_t id = n + lane < a.N ? a.ids[n + lane] : -1;
    uint64_t in = __ballot(id == (int32_t)v);
    any |= in != 0;
    while (in) {
      const int l = __ffsll((long long)in) - 1;
      in &= in - 1;
      add_rows<TI, 1, 1>(a, (int32_t)(n + l), 1, c, f);
    }
  }
  if (c >= a.H) return;
  if (any)
    store_sum<TO, 4>(a, v, c, f[0]);
  else if (!a.accumulate)  // (zeros, whatever the scale)
    store_wide<TO, 4, true>((char*)a.out + v * a.ldo * TO::BYTES, c, a.H, f[0]);
}

// Launches over rows (tokens, tiles, entries) in units of a row's chunk.
constexpr int64_t kEmbMaxUnits = ((int64_t)1 << 32) / kEmbThreads * kEmbWaves - kEmbWaves;
template <class Args, class F>
hipError_t launch_units(Args a, int64_t rows, int chunk, F launch) {
  const int64_t chunks = (a.H + chunk - 1) / chunk;
  a.chunks = (uint32_t)chunks;
  const int64_t most = kEmbMaxUnits / chunks;
  for (int64_t r0 = 0; r0 < rows; r0 += most) {
    const int64_t n = rows - r0 < most ? rows - r0 : most;
    a.row0 = r0;
    a.units = (uint32_t)(n * chunks);
    launch(a, dim3((unsigned)((a.units + kEmbWaves - 1) / kEmbWaves)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class TI, class TO>
hipError_t embed_t(const EmbedArgs& a, hipStream_t st) {
  constexpr int one = 64 * (16 / TO::BYTES);
#define OPD_EMBED(VPL)                                                                     \
  launch_units(a, a.N, one* VPL, [&](const EmbedArgs& b, dim3 g) {                         \
    hipLaunchKernelGGL((k_embed<TI, TO, VPL>), g, dim3(kEmbThreads), 0, st, b);            \
  })
  return a.H <= one ? OPD_EMBED(1) : a.H <= 2 * one ? OPD_EMBED(2) : OPD_EMBED(4);
#undef OPD_EMBED
}

template <class TI, class TO>
hipError_t embed_grad_t(EmbedGradArgs a, hipStream_t st) {
  if (!a.start)
    return launch_units(a, a.V, 256, [&](const EmbedGradArgs& b, dim3 g) {
      hipLaunchKernelGGL((k_embed_few<TI, TO>), g, dim3(kEmbThreads), 0, st, b);
    });
  hipLaunchKernelGGL(k_embed_group, dim3((unsigned)((a.V + a.keys - 1) / a.keys)),
                     dim3(kGroupThreads), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  a.tiles = (a.N + kEmbTile - 1) / kEmbTile;
#define OPD_SUMS(VPL)                                                                   \
  launch_units(a, a.tiles + a.N, 256 * VPL, [&](const EmbedGradArgs& b, dim3 g) {       \
    hipLaunchKernelGGL((k_embed_sums<TI, TO, VPL>), g, dim3(kEmbThreads), 0, st, b);    \
  })
  e = a.H <= 256 ? OPD_SUMS(1) : OPD_SUMS(2);
#undef OPD_SUMS
  if (e != hipSuccess) return e;
  // (added to: what has no token stays)
  return launch_units(a, a.tiles + (a.accumulate ? 0 : a.V), 64 * (16 / TO::BYTES),
                      [&](const EmbedGradArgs& b, dim3 g) {
                        hipLaunchKernelGGL((k_embed_rest<TO>), g, dim3(kEmbThreads), 0, st, b);
                      });
}

}  // namespace

hipError_t launch_embed(const EmbedArgs& a, int in_dt, int out_dt, hipStream_t st) {
  if (in_dt == BF16)
    return out_dt == BF16 ? embed_t<InBf16, OutBf16>(a, st) : embed_t<InBf16, OutF32>(a, st);
  return out_dt == BF16 ? embed_t<InF32, OutBf16>(a, st) : embed_t<InF32, OutF32>(a, st);
}

hipError_t launch_embed_grad(const EmbedGradArgs& a, int in_dt, int out_dt, hipStream_t st) {
  if (in_dt == BF16)
    return out_dt == BF16 ? embed_grad_t<InBf16, InBf16>(a, st) : embed_grad_t<InBf16, InF32>(a, st);
  return out_dt == BF16 ? embed_grad_t<InF32, InBf16>(a, st) : embed_grad_t<InF32, InF32>(a, st);
}

}  // namespace opd
