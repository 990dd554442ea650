// Tokens sorted by key (a vocabulary entry, an adapter), stably: those of a key
// in the order of the batch, so that sums over them are made in one fixed order.
// Internal; included by the .hip sources that need it.
#pragma once

#include "opd_device.h"

namespace opd {
namespace {

constexpr int kGroupThreads = 1024;
constexpr int kGroupWaves = kGroupThreads / 64;

template <int KEYS>  // of a workgroup, at most
struct GroupLds {
  uint32_t at[kGroupWaves][KEYS];  // tokens of a key in a wave's part; then where its next goes
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

// The lanes of `in` that hold lane's key, of `bits` bits.  Batches often lie packed, one key
// after the other: then the first comparison is all.
__device__ __forceinline__ uint64_t lanes_of_key(uint64_t in, int32_t k, int bits) {
  const int32_t one = __builtin_amdgcn_readlane(k, __ffsll((long long)in) - 1);
  if ((__ballot(k == one) & in) == in) return in;
  uint64_t same = in;
  for (int bit = 0; bit < bits; ++bit) {
    const int32_t mine = -(k >> bit & 1);  // (all bits, or none)
    const uint64_t b = __ballot(mine != 0);
    same &= ~(b ^ (uint64_t)(int64_t)mine);
  }
  return same;
}

// One workgroup sorts the tokens whose key lies in [lo, lo + count), count <=
// KEYS; key(n) of token n is < 2^31, or -1 for tokens that have no part.
// Two passes over all keys, a contiguous part of the tokens to each wave: counts
// per wave and key, then places.  The tokens of smaller keys are counted on the
// way, so workgroups need nothing of each other.  Writes perm for its keys;
// returns the first place of key lo + threadIdx.x (for lanes below count) and
// the place past the workgroup's last token.
template <int KEYS, bool FEW, class Key>
__device__ __forceinline__ uint32_t group_tokens(int64_t N, int32_t lo, int count, Key key,
                                                 int32_t* perm, GroupLds<KEYS>& sh, uint32_t& end) {
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int bits = 32 - __clz(count - 1 > 0 ? count - 1 : 1);
  if ((int)threadIdx.x < count) {
#pragma unroll
    for (int i = 0; i < kGroupWaves; ++i) sh.at[i][threadIdx.x] = 0;
  }
  __syncthreads();
  const int64_t part = (N + 64 * kGroupWaves - 1) / (64 * kGroupWaves) * 64;
  const int64_t n0 = w * part, n1 = n0 + part < N ? n0 + part : N;
  uint32_t below = 0;
  constexpr int A = 8;  // keys on their way at once; up to 64 A of a wave's stay in registers
  int32_t ks[A];
  uint64_t sames[A];
  const bool held = part <= 64 * A;
  auto load = [&](int64_t n) {
#pragma unroll
    for (int i = 0; i < A; ++i) ks[i] = key(min(n + 64 * i + lane, n1 - 1));
#pragma unroll
    for (int i = 0; i < A; ++i) ks[i] = n + 64 * i + lane < n1 ? ks[i] : -1;
  };
  for (int64_t n = n0; n < n1; n += 64 * A) {
    load(n);
#pragma unroll
    for (int i = 0; i < A; ++i) {
      if (ks[i] >= 0 && ks[i] < lo) ++below;
      const int32_t k = ks[i] - lo;
      const bool mine = ks[i] >= lo && k < count;
      if constexpr (FEW) {  // of all tokens are a workgroup's: they hardly meet
        if (mine) atomicAdd(&sh.at[w][k], 1u);
      } else {
        const uint64_t in = __ballot(mine);
        if (!in) continue;
        sames[i] = lanes_of_key(in, k, bits);
        if (mine && lane == __ffsll((long long)sames[i]) - 1)
          atomicAdd(&sh.at[w][k], (uint32_t)__popcll(sames[i]));
      }
    }
  }
  if (lo > 0) {
    below = (uint32_t)__shfl((int)wave_incl_scan_u32(below), 63, 64);
    if (lane == 0) sh.below[w] = below;
  }
  __syncthreads();
  uint32_t base = 0;
  if (lo > 0) {
#pragma unroll
    for (int i = 0; i < kGroupWaves; ++i) base += sh.below[i];
  }
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
  // A wave's tokens in order, 64 at a time: a lane finds those of its key by the keys'
  // bits, and the first of them takes their places.
  for (int64_t m = n0; m < n1; m += 64 * A) {
    if (!held) load(m);
#pragma unroll
    for (int i = 0; i < A; ++i) {
      const int32_t k = ks[i] - lo;
      const uint64_t all = __ballot(ks[i] >= lo && k < count);
      if (!all) continue;
      const uint64_t same = FEW || !held ? lanes_of_key(all, k, bits) : sames[i];
      if (all >> lane & 1) {
        const int lead = __ffsll((long long)same) - 1;
        uint32_t at = 0;
        if (lane == lead) at = atomicAdd(&sh.at[w][k], (uint32_t)__popcll(same));
        at = (uint32_t)__shfl((int)at, lead, 64) + (uint32_t)__popcll(same & ((1ull << lane) - 1));
        perm[at] = (int32_t)(m + 64 * i + lane);
      }
    }
  }
  return first;
}

}  // namespace
}  // namespace opd
