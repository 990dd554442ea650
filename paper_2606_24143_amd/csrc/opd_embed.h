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
constexpr int kEmbRows = 8;  // entries of a wavefront

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
// workgroup.  E: elements of a lane's store (16 bytes of it).
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

// Tokens sorted by id: start[v] the first place of entry v, perm the tokens.
__global__ void __launch_bounds__(kGroupThreads) k_embed_group(EmbedGradArgs a) {
  __shared__ GroupLds<kEmbKeys> sh;
  const int32_t lo = (int32_t)((int64_t)blockIdx.x * a.keys);
  const int count = (int)(a.V - lo < a.keys ? a.V - lo : a.keys);
  const int32_t* ids = a.ids;
  const int64_t V = a.V;
  uint32_t end;
  const uint32_t first = group_tokens(
      a.N, lo, count, [=](int64_t n) { return (uint32_t)ids[n] < (uint32_t)V ? ids[n] : -1; }, a.perm, sh, end);
  if ((int)threadIdx.x < count) a.start[lo + (int)threadIdx.x] = (int32_t)first;
  if (threadIdx.x == 0 && lo + count == a.V) a.start[a.V] = (int32_t)end;
}

// Adds dy[token, c0 ..] for the tokens that lanes [0, count) hold, in order; B rows on
// their way at once.
template <class TI, int VPL, int B>
__device__ __forceinline__ void add_rows(const EmbedGradArgs& a, int32_t token, int count,
                                         int64_t c0, float (&f)[VPL][4]) {
#pragma unroll 1
  for (int i = 0; i < count; i += B) {
    float x[B][VPL][4];
#pragma unroll
    for (int b = 0; b < B; ++b) {
      if (i + b >= count) continue;
      const char* row =
          (const char*)a.dy + (int64_t)__builtin_amdgcn_readlane(token, i + b) * a.ldy * TI::BYTES;
#pragma unroll
      for (int v = 0; v < VPL; ++v)
        if (c0 + v * 256 < a.H) load_wide<TI, 4>(row, c0 + v * 256, a.H, x[b][v]);
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

// Entries of more than kEmbTile tokens are summed tile by tile of the sorted
// tokens first, so that one frequent token does not keep one wavefront busy.  A
// tile holds a part of at most two such entries: one that begins before or at its
// first place (part 0), and one that begins inside it (part 1) and goes on past it.
constexpr int kEmbTile = 64;
template <class TI>
__global__ void __launch_bounds__(kEmbThreads) k_embed_tiles(EmbedGradArgs a) {
  const uint32_t u = blockIdx.x * kEmbWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int64_t tile = a.row0 + u / a.chunks;
  const int64_t p = tile * kEmbTile + lane;
  const int64_t kept = a.start[a.V];
  if (u >= a.units || tile * kEmbTile >= kept) return;
  const int64_t c0 = (int64_t)(u % a.chunks) * 256 + lane * 4;
  const int32_t token = p < kept ? a.perm[p] : 0;
  const int32_t id = p < kept ? a.ids[token] : -1;
  int32_t s = 0, e = 0;
  if (p < kept) {
    s = a.start[id];
    e = a.start[id + 1];
  }
  const bool many = e - s > kEmbTile;
#pragma unroll 1
  for (int part = 0; part < 2; ++part) {
    const uint64_t in = __ballot(many && (part == 0) == (s <= tile * kEmbTile));
    if (!in) continue;
    // (its places are consecutive: moved down to lane 0)
    const int first = __ffsll((long long)in) - 1, count = __popcll(in);
    const int32_t mine = __shfl(token, (first + lane) & 63, 64);
    float f[1][4] = {};
    add_rows<TI, 1, 16>(a, mine, count, c0, f);
    float* to = a.partial + (tile * 2 + part) * a.hp;
    if (c0 < a.H) *(f32x4*)(to + c0) = f32x4{f[0][0], f[0][1], f[0][2], f[0][3]};
  }
}

// One wavefront to kEmbRows entries and a chunk of 256 * VPL columns: first the entries
// without a token, which are stores alone, then the others': their tokens' rows, or their tiles'
// sums, in order.  SORTED false: no list; the wave looks for its entries' tokens
// among the ids itself (few tokens, one launch).
template <class TI, class TO, int VPL, bool SORTED>
__global__ void __launch_bounds__(kEmbThreads) k_embed_rows(EmbedGradArgs a) {
  const uint32_t block = xcd_eighths(blockIdx.x, gridDim.x);
  const uint32_t u = block * kEmbWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (u >= a.units) return;
  const int lane = threadIdx.x & 63;
  const int64_t v0 = (a.row0 + u / a.chunks) * kEmbRows;
  const int64_t c0 = (int64_t)(u % a.chunks) * (256 * VPL) + lane * 4;
  const int rows = (int)(a.V - v0 < kEmbRows ? a.V - v0 : kEmbRows);
  int32_t first = 0;
  uint64_t some = 0;  // bit i: entry v0 + i has a token
  if constexpr (SORTED) {
    first = a.start[v0 + (lane <= rows ? lane : rows)];
    const int32_t past = __shfl_down(first, 1, 64);
    some = __ballot(lane < rows && past > first);
  } else {
    for (int64_t n = 0; n < a.N; n += 64) {
      const int64_t id = n + lane < a.N ? (int64_t)a.ids[n + lane] - v0 : -1;
      uint64_t in = __ballot(id >= 0 && id < rows);
      while (in) {
        const int l = __ffsll((long long)in) - 1;
        in &= in - 1;
        some |= 1ull << __builtin_amdgcn_readlane((int)id, l);
      }
    }
  }
  auto out = [&](int i) { return (char*)a.out + (v0 + i) * a.ldo * TO::BYTES; };
  if (!a.accumulate) {
    const float zero[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int i = 0; i < rows; ++i) {
      if (some >> i & 1) continue;
#pragma unroll
      for (int v = 0; v < VPL; ++v)
        if (c0 + v * 256 < a.H) store_wide<TO, 4, true>(out(i), c0 + v * 256, a.H, zero);
    }
  }
#pragma unroll 1
  while (some) {
    const int i = __ffsll((long long)some) - 1;
    some &= some - 1;
    float f[VPL][4] = {};
    if constexpr (SORTED) {
      const int32_t s = __builtin_amdgcn_readlane(first, i);
      const int32_t e = __builtin_amdgcn_readlane(first, i + 1);
      if (e - s > kEmbTile) {
        const int64_t t1 = ((int64_t)e + kEmbTile - 1) / kEmbTile;
#pragma unroll 2
        for (int64_t t = s / kEmbTile; t < t1; ++t) {
          const float* from = a.partial + (t * 2 + (s > t * kEmbTile ? 1 : 0)) * a.hp;
#pragma unroll
          for (int v = 0; v < VPL; ++v) {
            if (c0 + v * 256 >= a.H) continue;
            const f32x4 x = *(const f32x4*)(from + c0 + v * 256);
#pragma unroll
            for (int k = 0; k < 4; ++k) f[v][k] += x[k];
          }
        }
      } else {
        add_rows<TI, VPL, 4>(a, lane < e - s ? a.perm[s + lane] : 0, e - s, c0, f);
      }
    } else {
      for (int64_t n = 0; n < a.N; n += 64) {
        const int64_t id = n + lane < a.N ? (int64_t)a.ids[n + lane] - v0 : -1;
        uint64_t in = __ballot(id == i);
        while (in) {
          const int l = __ffsll((long long)in) - 1;
          in &= in - 1;
          add_rows<TI, VPL, 1>(a, (int32_t)(n + l), 1, c0, f);
        }
      }
    }
    char* row = out(i);
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      if (c0 + v * 256 >= a.H) continue;
#pragma unroll
      for (int k = 0; k < 4; ++k) f[v][k] *= a.scale;
      if (a.accumulate) {
        float x[4];
        load_wide<TO, 4>(row, c0 + v * 256, a.H, x);
#pragma unroll
        for (int k = 0; k < 4; ++k) f[v][k] += x[k];
      }
      store_wide<TO, 4, true>(row, c0 + v * 256, a.H, f[v]);
    }
  }
}

// Launches over rows (tokens, tiles, groups of entries) in units of a row's chunk.
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

template <class TI, class TO, int VPL>
hipError_t embed_grad_v(const EmbedGradArgs& a, hipStream_t st) {
  const int64_t rows = (a.V + kEmbRows - 1) / kEmbRows;
  if (!a.start)
    return launch_units(a, rows, 256 * VPL, [&](const EmbedGradArgs& b, dim3 g) {
      hipLaunchKernelGGL((k_embed_rows<TI, TO, VPL, false>), g, dim3(kEmbThreads), 0, st, b);
    });
  hipLaunchKernelGGL(k_embed_group, dim3((unsigned)((a.V + a.keys - 1) / a.keys)),
                     dim3(kGroupThreads), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  e = launch_units(a, (a.N + kEmbTile - 1) / kEmbTile, 256, [&](const EmbedGradArgs& b, dim3 g) {
    hipLaunchKernelGGL((k_embed_tiles<TI>), g, dim3(kEmbThreads), 0, st, b);
  });
  if (e != hipSuccess) return e;
  return launch_units(a, rows, 256 * VPL, [&](const EmbedGradArgs& b, dim3 g) {
    hipLaunchKernelGGL((k_embed_rows<TI, TO, VPL, true>), g, dim3(kEmbThreads), 0, st, b);
  });
}

template <class TI, class TO>
hipError_t embed_grad_t(const EmbedGradArgs& a, hipStream_t st) {
  if (a.H <= 256) return embed_grad_v<TI, TO, 1>(a, st);
  if (a.H <= 512) return embed_grad_v<TI, TO, 2>(a, st);
  return embed_grad_v<TI, TO, 4>(a, st);
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
