// Tokens sorted by key (a vocabulary entry, an adapter), stably: those of a key
// in the order of the batch, so that sums over them are made in one fixed order.
// Internal; included by the .hip sources that need it.
#pragma once

#include "opd_device.h"

namespace opd {
namespace {

constexpr int kGroupThreads = 1024;
constexpr int kGroupWaves = kGroupThreads / 64;
constexpr int kGroupKeys = 1024;  // keys of a workgroup at most

struct GroupLds {
  uint32_t at[kGroupWaves][kGroupKeys];  // tokens of a key in a wave's part; then where its next goes
  uint32_t sums[kGroupWaves];
  uint32_t below[kGroupWaves];
};

__device__ __forceinline__ uint32_t wave_incl_scan_u32(uint32_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t t = (uint32_t)__shfl_up((int)v, o, 64);
    if (lane >= o) v += t;
  }
  return v;
}

// Exclusive sums over the workgroup's lanes, and the whole sum.
__device__ __forceinline__ uint32_t block_excl_scan(uint32_t v, uint32_t* sums, uint32_t& total) {
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const uint32_t incl = wave_incl_scan_u32(v);
  if (lane == 63) sums[w] = incl;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kGroupWaves; ++i) {
    before += i < w ? sums[i] : 0u;
    all += sums[i];
  }
  total = all;
  __syncthreads();
  return before + incl - v;
}

// One workgroup sorts the tokens whose key lies in [lo, lo + count), count <=
// kGroupKeys; key(n) of token n is < 2^31, or -1 for tokens that have no part.
// Two passes over all keys, a contiguous part of the tokens to each wave: counts
// per wave and key, then places.  The tokens of smaller keys are counted on the
// way, so workgroups need nothing of each other.  Writes perm for its keys;
// returns the first place of key lo + threadIdx.x (for lanes below count) and
// the place past the workgroup's last token.
template <class Key>
__device__ __forceinline__ uint32_t group_tokens(int64_t N, int32_t lo, int count, Key key,
                                                 int32_t* perm, GroupLds& sh, uint32_t& end) {
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int i = threadIdx.x; i < kGroupWaves * count; i += kGroupThreads)
    sh.at[i / count][i % count] = 0;
  __syncthreads();
  const int64_t part = (N + 64 * kGroupWaves - 1) / (64 * kGroupWaves) * 64;
  const int64_t n0 = w * part, n1 = n0 + part < N ? n0 + part : N;
  uint32_t below = 0;
  for (int64_t n = n0 + lane; n < n1; n += 64) {
    const int32_t k = key(n);
    if (k >= 0 && k < lo) ++below;
    if (k >= lo && k - lo < count) atomicAdd(&sh.at[w][k - lo], 1u);
  }
  below = (uint32_t)__shfl((int)wave_incl_scan_u32(below), 63, 64);
  if (lane == 0) sh.below[w] = below;
  __syncthreads();
  uint32_t base = 0;
#pragma unroll
  for (int i = 0; i < kGroupWaves; ++i) base += sh.below[i];
  uint32_t mine = 0;
  if ((int)threadIdx.x < count) {
#pragma unroll
    for (int i = 0; i < kGroupWaves; ++i) mine += sh.at[i][threadIdx.x];
  }
  uint32_t total;
  const uint32_t first = base + block_excl_scan(mine, sh.sums, total);
  if ((int)threadIdx.x < count) {
    uint32_t at = first;
#pragma unroll
    for (int i = 0; i < kGroupWaves; ++i) {
      const uint32_t c = sh.at[i][threadIdx.x];
      sh.at[i][threadIdx.x] = at;
      at += c;
    }
  }
  __syncthreads();
  end = base + total;
  // (a wave's tokens in order: 64 at a time, key by key)
  for (int64_t n = n0; n < n1; n += 64) {
    const int32_t k = n + lane < n1 ? key(n + lane) : -1;
    uint64_t left = __ballot(k >= lo && k - lo < count);
    while (left) {
      const int lead = __ffsll((long long)left) - 1;
      const int32_t kk = __builtin_amdgcn_readlane(k, lead);
      const uint64_t same = __ballot(k == kk);
      uint32_t at = 0;
      if (lane == lead) at = atomicAdd(&sh.at[w][kk - lo], (uint32_t)__popcll(same));
      at = (uint32_t)__builtin_amdgcn_readlane((int)at, lead);
      if (k == kk) perm[at + (uint32_t)__popcll(same & ((1ull << lane) - 1))] = (int32_t)(n + lane);
      left &= ~same;
    }
  }
  return first;
}

}  // namespace
}  // namespace opd
