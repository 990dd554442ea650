// The rows of logits themselves (Stages 1 and 2 read them; Sec. 4.1): hidden
// states and an output head in 8-bit floating point (e4m3: 3 bits of mantissa,
// values to 448) with a scale for each block of 128 columns, and their product.
// Internal; included by opd_cache_kernels.hip only.
//
//   quantise  a block's scale is its largest magnitude over 448 (fp32, or the
//             least power of two that is not below it), its values the nearest
//             e4m3 values of x / s;
//   product   z[n, v] = sum_b sx[n, b] sw[v / 128, b] sum_{h in b} x[n, h] w[v, h]
//             on the matrix cores, accumulated in fp32.
#pragma once

#include "opd_device.h"

namespace opd {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));

constexpr int kBlk = 128;          // columns of a block
constexpr float kTop = 448.0f;     // the largest e4m3 value
constexpr float kMinScale = 1.17549435e-38f;  // 2^-126

// ---------------------------------------------------------------- quantisation

// Eight consecutive elements of a row from column h on, as they are stored
// (columns past H read as 0).
template <class TI>
struct Eight {
  u32x4 v[TI::BYTES / 2];
};
template <class TI>
__device__ __forceinline__ Eight<TI> load8(const char* row, int64_t h, int64_t H) {
  Eight<TI> r;
  const u32x4* p = (const u32x4*)(row + h * TI::BYTES);
  if (h + 8 <= H) {
#pragma unroll
    for (int d = 0; d < TI::BYTES / 2; ++d) r.v[d] = __builtin_nontemporal_load(p + d);
  } else {
#pragma unroll
    for (int d = 0; d < TI::BYTES / 2; ++d) r.v[d] = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (h + e >= H) continue;
      if constexpr (TI::BYTES == 2)
        r.v[0][e / 2] |= (uint32_t)((const uint16_t*)row)[h + e] << (16 * (e & 1));
      else
        r.v[e / 4][e & 3] = ((const uint32_t*)row)[h + e];
    }
  }
  return r;
}
template <class TI>
__device__ __forceinline__ float elem8(const Eight<TI>& x, int e) {
  if constexpr (TI::BYTES == 2)
    return __uint_as_float(e & 1 ? x.v[0][e / 2] & 0xFFFF0000u : x.v[0][e / 2] << 16);
  else
    return __uint_as_float(x.v[e / 4][e & 3]);
}
// The largest magnitude as bits: an integer maximum, in which a NaN is above an
// infinity and both above every number, so neither is lost.
template <class TI>
__device__ __forceinline__ uint32_t top8(const Eight<TI>& x, uint32_t top) {
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(elem8<TI>(x, e)) & 0x7FFFFFFFu);
  return top;
}

struct Scale {
  float s;        // what values are divided by (NaN: the block holds a NaN or an infinity)
  float inv;      // 1 / s (e8m0: exact)
  uint32_t e8m0;  // its biased exponent (255: NaN)
};

template <bool E8>
__device__ __forceinline__ Scale block_scale(uint32_t top) {
  Scale r;
  const bool bad = top >= 0x7F800000u;
  r.e8m0 = 255u;
  if constexpr (E8) {
    // 448 = 1.75 * 2^8: a = m 2^e needs 2^(e - 8), or 2^(e - 7) for m > 1.75.
    // (a below 2^-126 has e = -127 in its bits and gets the least power.)
    int e = (int)(top >> 23) - 127 - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    e = e < -127 ? -127 : e;
    if (!bad) r.e8m0 = (uint32_t)(e + 127);
    r.s = bad ? __builtin_nanf("") : ldexpf(1.0f, e);
    r.inv = ldexpf(1.0f, -e);
  } else {
    r.s = bad ? __builtin_nanf("") : fmaxf(__uint_as_float(top) / kTop, kMinScale);
    r.inv = 1.0f / r.s;
  }
  return r;
}

// f / s, correctly rounded (its last bit decides the ties of the 8-bit rounding).
// A power of two's inverse is exact.  Else two corrections of f times the rounded
// inverse, by their exact remainders: the first leaves less than a step, from which
// the second gives the rounded quotient (Markstein, IBM J. Res. Dev. 34(1), 1990).
// Five instructions for a division's eleven; where the remainders of such values
// could underflow (s below 2^-60) it divides.  (The remainders are q s - f, which is
// +0 where f is -0: taken from q it leaves -0.  f - q s, added, would leave +0.)
constexpr float kSmallScale = 8.6736174e-19f;  // 2^-60
template <bool E8>
__device__ __forceinline__ float quotient(float f, const Scale& sc, bool small) {
  if constexpr (E8) return f * sc.inv;
  if (small) return f / sc.s;
  float q = f * sc.inv;
  q = fmaf(fmaf(q, sc.s, -f), -sc.inv, q);
  return fmaf(fmaf(q, sc.s, -f), -sc.inv, q);
}

// The nearest e4m3 values of f / s, eight to a lane, packed.
template <class TI, bool E8>
__device__ __forceinline__ u32x2 quant8(const Eight<TI>& x, const Scale& sc) {
  const bool small = !E8 && __ballot(!(sc.s >= kSmallScale)) != 0;
  float v[8];
  if (small) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = quotient<E8>(elem8<TI>(x, e), sc, true);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = quotient<E8>(elem8<TI>(x, e), sc, false);
  }
  u32x2 r;
#pragma unroll
  for (int d = 0; d < 2; ++d) {
    int w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * d], v[4 * d + 1], w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * d + 2], v[4 * d + 3], w, true);
    r[d] = sc.s == sc.s ? (uint32_t)w : 0x7F7F7F7Fu;
  }
  return r;
}

__device__ __forceinline__ void store8(uint8_t* qrow, int64_t h, int64_t H, u32x2 q) {
  if (h + 8 <= H) {
    __builtin_nontemporal_store(q, (u32x2*)(qrow + h));
  } else {
    for (int e = 0; h + e < H; ++e) qrow[h + e] = (uint8_t)(q[e >> 2] >> (8 * (e & 3)));
  }
}

template <bool E8>
__device__ __forceinline__ void store_scale(void* scales, int64_t at, const Scale& s) {
  if constexpr (E8)
    ((uint8_t*)scales)[at] = (uint8_t)s.e8m0;
  else
    ((float*)scales)[at] = s.s;
}

// Blocks of one row: 16 lanes, eight elements each, to a block; the 16 lanes take
// QB consecutive blocks (of the rows one after the other), both loaded first.  Bound
// by HBM: 8,192 x 4,096 bf16, e8m0, 101 MB in 17.6 us (5.7 TB/s, part of it from the
// Infinity Cache; 23 us with a block at a time).
constexpr int kQuantThreads = 256;
template <class TI, bool E8, int QB>
__global__ void __launch_bounds__(kQuantThreads) k_quantize_rows(QuantArgs a, int64_t first) {
  const int64_t blocks = a.N * a.nb;
  const int64_t g0 = first + ((int64_t)blockIdx.x * (kQuantThreads / 16) + (threadIdx.x >> 4)) * QB;
  if (g0 >= blocks) return;
  int64_t row = g0 / a.nb, b = g0 - row * a.nb;
  Eight<TI> x[QB];
  int64_t rows[QB], h[QB];
#pragma unroll
  for (int k = 0; k < QB; ++k) {
    rows[k] = row;
    h[k] = b * kBlk + 8 * (threadIdx.x & 15);
    if (g0 + k < blocks)
      x[k] = load8<TI>((const char*)a.x + row * a.ldx * TI::BYTES, h[k], a.H);
    if (++b == a.nb) {
      b = 0;
      ++row;
    }
  }
#pragma unroll
  for (int k = 0; k < QB; ++k) {
    if (g0 + k >= blocks) break;
    uint32_t top = top8<TI>(x[k], 0u);
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
    const Scale s = block_scale<E8>(top);
    store8(a.q + rows[k] * a.ldq, h[k], a.H, quant8<TI, E8>(x[k], s));
    if ((threadIdx.x & 15) == 0) store_scale<E8>(a.scales, g0 + k, s);
  }
}

// A block of 128 rows: a workgroup, eight passes of 16 rows held in registers, so x
// is read once.  Bound by HBM and, with fp32 scales, by the quotients beside it:
// 151,936 x 4,096 bf16, 1,867 MB in 313 us (6.0 TB/s; divisions made it 390).
template <class TI, bool E8>
__global__ void __launch_bounds__(kQuantThreads) k_quantize_tiles(QuantArgs a, int64_t first) {
  __shared__ uint32_t red[kQuantThreads / 64];
  const int64_t at = first + blockIdx.x;
  const int64_t br = at / a.nb, b = at - br * a.nb;
  const int64_t h = b * kBlk + 8 * (threadIdx.x & 15);
  const int64_t r0 = br * kBlk + (threadIdx.x >> 4);
  Eight<TI> x[8];
  uint32_t top = 0;
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const int64_t row = min(r0 + 16 * p, a.N - 1);  // (the last row again: the same maximum)
    x[p] = load8<TI>((const char*)a.x + row * a.ldx * TI::BYTES, h, a.H);
  }
#pragma unroll
  for (int p = 0; p < 8; ++p) top = top8<TI>(x[p], top);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kQuantThreads / 64; ++w) top = max(top, red[w]);
  const Scale s = block_scale<E8>(top);
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const int64_t row = r0 + 16 * p;
    if (row < a.N) store8(a.q + row * a.ldq, h, a.H, quant8<TI, E8>(x[p], s));
  }
  if (threadIdx.x == 0) store_scale<E8>(a.scales, at, s);
}

// (a launch has fewer than 2^32 work-items: larger calls are several)
constexpr int64_t kMaxGroups = 0xFFFFFFFFll / kQuantThreads;

template <class TI, bool E8>
hipError_t launch_quantize_t(const QuantArgs& a, hipStream_t stream) {
  constexpr int QB = 2;
  const bool rows = a.block_rows == 1;
  const int64_t blocks = (rows ? a.N : (a.N + kBlk - 1) / kBlk) * a.nb;
  const int64_t per = rows ? kQuantThreads / 16 * QB : 1;  // blocks of a workgroup
  for (int64_t first = 0; first < blocks; first += kMaxGroups * per) {
    const int64_t groups = min((blocks - first + per - 1) / per, kMaxGroups);
    if (rows)
      hipLaunchKernelGGL((k_quantize_rows<TI, E8, QB>), dim3((unsigned)groups), dim3(kQuantThreads),
                         0, stream, a, first);
    else
      hipLaunchKernelGGL((k_quantize_tiles<TI, E8>), dim3((unsigned)groups), dim3(kQuantThreads), 0,
                         stream, a, first);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ---------------------------------------------------------------- product

// 2^(e - 127) (2^-127 is not a normal number; 255 is NaN)
__device__ __forceinline__ float e8m0_value(uint32_t e) {
  return e == 255u ? __builtin_nanf("") : __uint_as_float(e ? e << 23 : 0x400000u);
}
// Four logits of consecutive vocabulary entries v .. v + 3 of one token.
template <class TO>
__device__ __forceinline__ void store_logits(void* row, int64_t v, int64_t V, f32x4 z) {
  if (v + 4 <= V) {
    if constexpr (TO::BYTES == 4)
      *(f32x4*)((float*)row + v) = z;
    else
      *(u32x2*)((uint16_t*)row + v) = u32x2{pack_bf16x2(z[0], z[1]), pack_bf16x2(z[2], z[3])};
  } else {
    for (int e = 0; v + e < V; ++e) {
      if constexpr (TO::BYTES == 4)
        ((float*)row)[v + e] = z[e];
      else
        ((uint16_t*)row)[v + e] = __builtin_bit_cast(uint16_t, (__bf16)z[e]);
    }
  }
}

// Eight e4m3 values as bf16, which holds them exactly.
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ bf16x8 widen8(int lo, int hi) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The 8-bit instruction cuts each product at 2^-13 of the largest of the 16 it sums
// at once before they reach the fp32 accumulator (measured: 1.5e-5 of a result
// of 64 normal products; the 16-bit instructions: 5e-9).  That is below the rounding of
// bf16 logits: 4,096 tokens, V = 151,936, H = 4,096, some channels of the hidden states
// far larger than the others, lie 1.6589e-3 of their norm from the exact logits, and
// exact products rounded to bf16 1.6588e-3 (they differ in one logit of 80, by a
// step).  It is not below that of fp32 ones, so these are made by 16-bit instructions
// of exactly widened values, at half the rate.  (bf16 logits from these as well, V =
// 151,936, H = 4,096, fp32 scales, us: 1 token 116 / 117, 32 119 / 121, 64 135 / 150, 128
// 179 / 235.  All take the 8-bit ones, so that a token's logits do not depend on how
// many are asked for with it by more than the order of sums.)
// 16 rows over 128 columns, of which a lane holds 32: as the instructions for TO take
// them; and the product of two.
template <class TO>
struct Frag {
  i32x8 v;
  __device__ __forceinline__ explicit Frag(i32x8 x) : v(x) {}
  Frag() = default;
};
template <>
struct Frag<OutF32> {
  bf16x8 v[4];
  __device__ __forceinline__ explicit Frag(i32x8 x) {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = widen8(x[2 * k], x[2 * k + 1]);
  }
  Frag() = default;
};
template <class TO>
__device__ __forceinline__ f32x4 mma128(const Frag<TO>& w, const Frag<TO>& x) {
  f32x4 c = {0.f, 0.f, 0.f, 0.f};
  if constexpr (TO::BYTES == 2) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.v, x.v, c, 0, 0, 0, 0, 0, 0);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.v[k], x.v[k], c, 0, 0, 0);
    return c;
  }
}

// Eight logits of consecutive entries from v on of one token.
template <class TO>
__device__ __forceinline__ void store8_logits(char* row, int64_t v, int64_t V, f32x4 a, f32x4 b) {
  if constexpr (TO::BYTES == 2) {
    if (v + 8 <= V) {
      *(u32x4*)((uint16_t*)row + v) = u32x4{pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]),
                                            pack_bf16x2(b[0], b[1]), pack_bf16x2(b[2], b[3])};
      return;
    }
  }
  store_logits<TO>(row, v, V, a);
  store_logits<TO>(row, v + 4, V, b);
}

// What is kept of 16 bytes of a row from byte h on: those before H.
__device__ __forceinline__ u32x4 keep16(u32x4 x, int h, int H) {
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const int n = H - h - 4 * d;  // valid bytes from this dword on
    x[d] = n >= 4 ? x[d] : n > 0 ? x[d] & ((1u << (8 * n)) - 1u) : 0u;
  }
  return x;
}

__device__ __forceinline__ uint32_t key_x(uint32_t row) { return (row >> 1) & 7u; }
__device__ __forceinline__ uint32_t key_w(uint32_t row) {
  return ((row >> 1) & 1u) | ((row >> 2) & 6u);
}

// bytes of rows from p on (none if bytes <= 0); reads past them give zeros
__device__ __forceinline__ Rsrc rows_rsrc(const void* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0,
                                           (int)(uint32_t)(bytes > 0 ? bytes : 0), kRsrcWord3);
}

// ---- few tokens
// Of few tokens the product is a read of the head.  W waves of 16 of its rows each,
// 128 tokens at most (T groups of 16; of more, blockIdx.y's).  The head goes from memory to the matrix
// instructions' registers, SB blocks ahead; the tokens through LDS, SB blocks a
// stage, shared by the waves.  Workgroups start at different stages of the rows:
// rows are often a multiple of 4 KiB apart, and all reads at one place of them wait
// for the same part of the memory (127 against 137 us at 32 tokens, V = 151,936, H =
// 4,096; 27 against 30 at 16, V = 32,000).  At V = 151,936, H = 4,096 (622 MB): 1 token
// 112 us (5.6 TB/s), 32 120, 64 135, 128 178; reads alone in this order take 100.  Two
// groups of rows to a wave, which halve the reads of LDS, gave 139 for 64.
template <class TO, bool E8, bool ODD, int T, int SB, int W>
__global__ void __launch_bounds__(64 * W, 2) k_head_stream(HeadArgs a) {
  constexpr bool HW = E8 && TO::BYTES == 2;
  constexpr int SZ = E8 ? 1 : 4, THREADS = 64 * W;
  constexpr int ROWS = 16 * T, PIECES = ROWS * SB * 8, PER = (PIECES + THREADS - 1) / THREADS;
  constexpr int SPER = (ROWS * SB + THREADS - 1) / THREADS;
  __shared__ __align__(16) uint8_t lx[2][SB][ROWS * 128];
  __shared__ uint32_t lsc[2][SB][ROWS];
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t lr = (uint32_t)lane & 15u, lk = (uint32_t)lane >> 4;
  const int64_t v0 = ((int64_t)blockIdx.x * W + w) * 16;
  const int64_t n0 = (int64_t)blockIdx.y * ROWS;  // the launch's tokens are 16 T at a time
  a.x += n0 * a.ldx;
  a.sx = (const char*)a.sx + n0 * a.nb * SZ;
  a.out = (char*)a.out + n0 * a.ldo * TO::BYTES;
  a.N = min(a.N - n0, (int64_t)ROWS);
  const uint32_t ldw = (uint32_t)a.ldw, ldx = (uint32_t)a.ldx;
  const int64_t vr = min(v0, a.V - 1);  // (a wave past the last row reads nothing)
  const uint8_t* gw = a.w + vr * a.ldw;
  const int64_t wbytes = v0 < a.V ? min((int64_t)16, a.V - v0) * a.ldw : 0;
  const int64_t xbytes = a.N * a.ldx;
  const int sbytes = (int)a.N * a.nb * SZ;
  const uint8_t* gh = (const uint8_t*)a.sw + (vr / kBlk) * a.nb * SZ;  // (16 divides 128)
  const uint32_t ow = lr * ldw + lk * 16;

  u32x4 px[PER];
  uint32_t ps[SPER], hs[SB];
  i32x8 bw[SB];
  // (`more`: no stage is read twice, which the last ones would be)
  auto ask_x = [&](int b0, bool more) {
    const Rsrc q =
        rows_rsrc(a.x + (int64_t)b0 * kBlk, more ? xbytes - (int64_t)b0 * kBlk : 0);
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const uint32_t i = (uint32_t)tid + k * THREADS, at = i & (SB * 8 - 1), row = i / (SB * 8);
      const bool in = b0 * kBlk + (int)at * 16 < (int)a.H && (PIECES % THREADS == 0 || i < PIECES);
      px[k] = __builtin_amdgcn_raw_buffer_load_b128(q, in ? (int)(row * ldx + at * 16) : INT32_MIN,
                                                    0, 0);
    }
    const Rsrc qs = rows_rsrc((const uint8_t*)a.sx + b0 * SZ, more ? sbytes - b0 * SZ : 0);
#pragma unroll
    for (int k = 0; k < SPER; ++k) {
      const uint32_t i = (uint32_t)tid + k * THREADS, row = i / SB, b = i & (SB - 1);
      const int o = b0 + (int)b < a.nb && row < ROWS ? (int)((row * a.nb + b) * SZ) : INT32_MIN;
      if constexpr (E8)
        ps[k] = __builtin_amdgcn_raw_buffer_load_b8(qs, o, 0, 0);
      else
        ps[k] = __builtin_amdgcn_raw_buffer_load_b32(qs, o, 0, 0);
    }
  };
  auto put_x = [&](int buf, int b0) {
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const uint32_t i = (uint32_t)tid + k * THREADS, at = i & (SB * 8 - 1), row = i / (SB * 8);
      if (ODD) px[k] = keep16(px[k], b0 * kBlk + (int)at * 16, (int)a.H);
      if (PIECES % THREADS == 0 || i < PIECES)
        *(u32x4*)(lx[buf][at >> 3] + row * 128 + (((at & 7u) ^ key_x(row)) << 4)) = px[k];
    }
#pragma unroll
    for (int k = 0; k < SPER; ++k) {
      const uint32_t i = (uint32_t)tid + k * THREADS, row = i / SB;
      if (row < ROWS) lsc[buf][i & (SB - 1)][row] = ps[k];
    }
  };
  auto ask_w = [&](int d, int b, bool more) {
    const int h = b * kBlk + (int)lk * 16;
    const bool in0 = h < (int)a.H, in1 = h + 64 < (int)a.H;
    const Rsrc q = rows_rsrc(gw + (int64_t)b * kBlk, more ? wbytes - (int64_t)b * kBlk : 0);
    const u32x4 lo = __builtin_amdgcn_raw_buffer_load_b128(q, in0 ? (int)ow : INT32_MIN, 0, 0);
    const u32x4 hi =
        __builtin_amdgcn_raw_buffer_load_b128(q, in1 ? (int)(ow + 64) : INT32_MIN, 0, 0);
    bw[d] = __builtin_bit_cast(i32x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    const Rsrc qs = rows_rsrc(gh + b * SZ, more && b < a.nb ? SZ : 0);
    if constexpr (E8)
      hs[d] = __builtin_amdgcn_raw_buffer_load_b8(qs, 0, 0, 0);
    else
      hs[d] = __builtin_amdgcn_raw_buffer_load_b32(qs, 0, 0, 0);
  };
  f32x4 acc[T];
#pragma unroll
  for (int t = 0; t < T; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const uint32_t fx0 = lr * 128 + ((lk ^ key_x(lr)) << 4);
  auto multiply = [&](int d, int buf, int b) {
    if (ODD) {
      const int h = b * kBlk + (int)lk * 16;
      const u32x4 lo = keep16(__builtin_shufflevector(__builtin_bit_cast(u32x8, bw[d]),
                                                      __builtin_bit_cast(u32x8, bw[d]), 0, 1, 2, 3),
                              h, (int)a.H);
      const u32x4 hi = keep16(__builtin_shufflevector(__builtin_bit_cast(u32x8, bw[d]),
                                                      __builtin_bit_cast(u32x8, bw[d]), 4, 5, 6, 7),
                              h + 64, (int)a.H);
      bw[d] = __builtin_bit_cast(i32x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    const Frag<TO> head(bw[d]);
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const uint8_t* p = lx[buf][d] + t * 2048;
      const i32x4 lo = *(const i32x4*)(p + fx0), hi = *(const i32x4*)(p + (fx0 ^ 64u));
      const i32x8 x = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      const uint32_t ts = lsc[buf][d][16 * t + lr];
      if constexpr (HW) {
        acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(bw[d], x, acc[t], 0, 0, 0,
                                                                  (int)hs[d], 0, (int)ts);
      } else {
        const float s = E8 ? e8m0_value(ts) * e8m0_value(hs[d])
                           : __uint_as_float(ts) * __uint_as_float(hs[d]);
        const f32x4 q = mma128<TO>(head, Frag<TO>(x));
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[t][e] = fmaf(q[e], s, acc[t][e]);
        // (added here, not kept for later: the products would fill the registers)
        if (T > 1) asm volatile("" : "+v"(acc[t]));
      }
      if (T > 2) __builtin_amdgcn_sched_barrier(0);
    }
  };
  // stages in a cycle that starts elsewhere for each workgroup
  const int stages = (a.nb + SB - 1) / SB;
  int now = (int)(blockIdx.x % (uint32_t)stages);  // the stage that is multiplied
  auto after = [&](int at) { return at + 1 == stages ? 0 : at + 1; };
  ask_x(now * SB, true);
#pragma unroll
  for (int d = 0; d < SB; ++d) ask_w(d, now * SB + d, true);
  put_x(0, now * SB);
  ask_x(after(now) * SB, stages > 1);
  int buf = 0;
  for (int i = 0; i < stages; ++i, buf ^= 1) {
    __syncthreads();
    const int next = after(now);
#pragma unroll
    for (int d = 0; d < SB; ++d) {
      multiply(d, buf, now * SB + d);
      ask_w(d, next * SB + d, i + 1 < stages);
      __builtin_amdgcn_sched_barrier(0);
      if (d == SB - 1) {
        put_x(buf ^ 1, next * SB);
        ask_x(after(next) * SB, i + 2 < stages);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    now = next;
  }
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const int64_t token = 16 * t + lr;
    if (token < a.N)
      store_logits<TO>((char*)a.out + token * a.ldo * TO::BYTES, v0 + 4 * lk, a.V, acc[t]);
  }
}

template <class TO, bool E8, int T, int SB, int W>
hipError_t launch_stream(const HeadArgs& a, hipStream_t stream) {
  const auto kernel = a.H % 16 != 0 ? k_head_stream<TO, E8, true, T, SB, W>
                                    : k_head_stream<TO, E8, false, T, SB, W>;
  hipLaunchKernelGGL(kernel,
                     dim3((unsigned)((a.V + 16 * W - 1) / (16 * W)),
                          (unsigned)((a.N + 16 * T - 1) / (16 * T))),
                     dim3(64 * W), 0, stream, a);
  return hipGetLastError();
}

// Waves to a workgroup: many share their tokens, few spread a narrow head over the
// CUs.  Measured, 2 / 4 / 8 waves, us: 1 token, V = 8,000, H = 4,096 10.8 / 13.8 / 21.1;
// 32,000 x 2,048 - / 13.4 / 15.1; 32 tokens, 4,000 x 4,096 10.5 / 11.6 / 19.6;
// 16,000 x 2,048 9.1 / 9.1 / 12.0; 32,000 x 4,096 34.2 / 30.5 / 28.4; 64 tokens, 4,000 18.8 /
// 17.5 / 23.5; 16,000 x 2,048 14.3 / 11.5 / 14.4; 64,000 x 4,096 95.0 / 69.8 / 61.3.
// Both scales and both types of logits agree to a tenth, and so do widths: 4 / 8 waves, 32
// tokens x 128,256 at H = 2,048 57 / 58, 5,120 135 / 123, 7,168 179 / 164, 16,384 441 / 358;
// not 8,192, 203 / 265 (32,000 entries 53 / 71), for a reason that is not known.  Between the
// bounds up to a quarter is lost (32 tokens x 12,000 x 4,096, fp32 logits 19.6 / 15.8 / 21.3).
template <class TO, bool E8>
hipError_t launch_few(const HeadArgs& a, hipStream_t stream) {
  const bool narrow = a.V < 12288, wide = a.V >= 24576;
  if (a.N <= 16)
    return narrow ? launch_stream<TO, E8, 1, 4, 2>(a, stream)
                  : launch_stream<TO, E8, 1, 4, 4>(a, stream);
  if (a.N <= 32)
    return narrow ? launch_stream<TO, E8, 2, 4, 2>(a, stream)
           : wide ? launch_stream<TO, E8, 2, 4, 8>(a, stream)
                  : launch_stream<TO, E8, 2, 4, 4>(a, stream);
  if (a.N <= 64)
    return wide ? launch_stream<TO, E8, 4, 4, 8>(a, stream)
                : launch_stream<TO, E8, 4, 4, 4>(a, stream);
  return launch_stream<TO, E8, 8, 2, 8>(a, stream);
}

// ---- many tokens
// A tile of 256 vocabulary entries by 256 tokens, eight waves of 128 by 64, one
// workgroup per CU that stays for all its tiles.  A block of 128 columns is a
// stage: 64 KiB in LDS, twice.  While the waves multiply stage g, each thread moves
// its eight pieces of stage g + 1 from registers to LDS and asks for those of stage
// g + 2, a piece to a slice of the products (all at once they fill the queues
// of the LDS and the address unit, and the matrix cores wait: 2.55 against 2.30
// ms, e8m0, at 4,096 tokens, V = 151,936, H = 4,096).  The stages of the next tile
// follow those of this one without a gap.
//
// The vocabulary is the matrix instructions' row index, so a lane's results are
// consecutive entries of one token, and its scales one per 16 tokens; the head's
// scale is the wave's.  e8m0 scales go to the instructions; fp32 ones multiply
// each block's product as it is added to the sum, which costs the vector unit
// half the matrix cores' time.  At that size e8m0 scales take 2.11-2.36 ms (2.3
// PFLOP/s; the matrix cores are busy for 61% of it), fp32 ones 2.55-2.74 (50%): what is
// left is the barrier of a stage, at which no other workgroup fills the CU.  fp32
// logits: 4.7 ms; 1,111 tokens, V = 50,257, H = 2,000 252-277 us (0.8 PFLOP/s at the
// 16-bit instructions' rate; 985 tiles on 256 CUs are four rounds).
//
// LDS rows are 128 bytes, 16-byte pieces at piece ^ key(row): with the keys below
// the 16 rows that a fragment read takes at once lie in different banks.  A fragment
// is pieces k and k + 4 of a row (k: the lane's quarter of the wave): which columns a
// lane holds does not matter as long as both operands agree.  Rows of the head are
// read in an order that leaves a lane eight consecutive entries from two products.
constexpr int kTileV = 256, kTileN = 256, kTileThreads = 512;
constexpr uint32_t kHeadCus = 256;
constexpr int kGroupV = 8;  // vocabulary tiles that take turns, so that rows of x stay in L2

template <bool E8>
struct HeadTile {  // where a tile's operands are (wave-uniform)
  static constexpr int SB = E8 ? 1 : 4;
  const uint8_t *w, *x, *s;
  int64_t wbytes, xbytes;
  int sbytes;
  int64_t v0, n0;
  // tile t of the launch; past its last one, a tile without rows
  __device__ __forceinline__ HeadTile(const HeadArgs& a, uint32_t t, uint32_t tiles, bool scales_w) {
    const uint32_t vtiles = (uint32_t)((a.V + kTileV - 1) / kTileV), nt = (uint32_t)a.ntiles;
    const bool is = t < tiles;
    t = is ? t : 0u;
    const uint32_t per = kGroupV * nt, g = t / per, r = t - g * per;
    const uint32_t gv = min((uint32_t)kGroupV, vtiles - g * kGroupV);
    v0 = (int64_t)(g * kGroupV + r % gv) * kTileV;
    n0 = (int64_t)(r / gv) * kTileN;
    w = a.w + v0 * a.ldw;
    x = a.x + n0 * a.ldx;
    wbytes = is ? min((int64_t)kTileV, a.V - v0) * a.ldw : 0;
    xbytes = is ? min((int64_t)kTileN, a.N - n0) * a.ldx : 0;
    // scales: of the tokens, or of the tile's two blocks of the head
    const int64_t s0 = scales_w ? v0 / kBlk : n0;
    const int64_t srows = scales_w ? min((int64_t)2, (a.V + kBlk - 1) / kBlk - s0)
                                   : min((int64_t)kTileN, a.N - n0);
    s = (const uint8_t*)(scales_w ? a.sw : a.sx) + s0 * a.nb * SB;
    sbytes = is ? (int)srows * a.nb * SB : 0;
  }
};

template <class TO, bool E8, bool ODD>
__global__ void __launch_bounds__(kTileThreads, 2) k_head_tile(HeadArgs a) {
  constexpr bool WIDE = TO::BYTES == 4;  // 16-bit instructions (mma128)
  constexpr bool HW = E8 && !WIDE;       // the instructions apply the scales
  constexpr int JH = HW ? 4 : 2;         // groups of 16 tokens at a time
  constexpr int PF = 2;                  // fragments of the head on the way
  constexpr int FIRST = HW ? 0 : 1;      // the first slice that moves a piece
  __shared__ __align__(16) uint8_t lds[2][2][256 * 128];  // [stage][head, tokens]
  __shared__ uint32_t lsc[2][kTileN + 2];                 // tokens' scales, then the head's
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t tiles = (uint32_t)(((a.V + kTileV - 1) / kTileV) * a.ntiles);
  // workgroups of XCD k (every eighth) share its contiguous part of the tiles
  const uint32_t G = gridDim.x, xcds = min(G, (uint32_t)kXcds);
  const uint32_t xcd = blockIdx.x % xcds, mine = blockIdx.x / xcds;
  const uint32_t step = (G - xcd + xcds - 1) / xcds;
  const uint32_t t1 = (uint32_t)((uint64_t)tiles * (xcd + 1) / xcds);
  uint32_t t = (uint32_t)((uint64_t)tiles * xcd / xcds) + mine;
  if (t >= t1) return;

  const int wv = (w & 1) * 128, wn = (w >> 1) * 64;
  const uint32_t ldw = (uint32_t)a.ldw, ldx = (uint32_t)a.ldx;
  const uint32_t prow = (uint32_t)tid >> 3, piece = (uint32_t)tid & 7u;
  const uint32_t ow = prow * ldw + piece * 16, ox = prow * ldx + piece * 16;
  const uint32_t os = (uint32_t)(tid & 255) * a.nb * HeadTile<E8>::SB;
  // (rows 64 apart have the same keys)
  const uint32_t ww = prow * 128 + ((piece ^ key_w(prow)) << 4);
  const uint32_t wx = prow * 128 + ((piece ^ key_x(prow)) << 4);
  const uint32_t lr = (uint32_t)lane & 15u, lk = (uint32_t)lane >> 4;
  const uint32_t rw = 8 * (lr >> 2) + (lr & 3);  // the head's row in a pair of products
  const uint32_t fw0 = rw * 128 + ((lk ^ key_w(rw)) << 4);
  const uint32_t fx0 = lr * 128 + ((lk ^ key_x(lr)) << 4);

  u32x4 pw[4], px[4];  // the pieces on their way
  uint32_t psc = 0;
  auto ask = [&](const HeadTile<E8>& h, int b, int k) {
    // (a piece past the row's end: past the buffer's, which gives zeros)
    const bool in = b * kBlk + (int)piece * 16 < (int)a.H;
    if (k < 4) {
      const Rsrc r = rows_rsrc(h.w + b * kBlk, h.wbytes - b * kBlk);
      pw[k] = __builtin_amdgcn_raw_buffer_load_b128(
          r, in ? (int)(ow + (uint32_t)k * 64 * ldw) : INT32_MIN, 0, 0);
    } else {
      const Rsrc r = rows_rsrc(h.x + b * kBlk, h.xbytes - b * kBlk);
      px[k - 4] = __builtin_amdgcn_raw_buffer_load_b128(
          r, in ? (int)(ox + (uint32_t)(k - 4) * 64 * ldx) : INT32_MIN, 0, 0);
    }
    if (k == 0) {
      const Rsrc r = rows_rsrc(h.s + b * HeadTile<E8>::SB, h.sbytes - b * HeadTile<E8>::SB);
      if constexpr (E8)
        psc = __builtin_amdgcn_raw_buffer_load_b8(r, b < a.nb ? (int)os : INT32_MIN, 0, 0);
      else
        psc = __builtin_amdgcn_raw_buffer_load_b32(r, b < a.nb ? (int)os : INT32_MIN, 0, 0);
    }
  };
  auto put = [&](int buf, int k) {
    if (k < 4)
      *(u32x4*)(lds[buf][0] + ww + k * 8192) = pw[k];
    else
      *(u32x4*)(lds[buf][1] + wx + (k - 4) * 8192) = px[k - 4];
    if (k == 0 && tid < kTileN + 2) lsc[buf][tid] = psc;
  };
  auto frag_w = [&](const uint8_t* base, int i) {
    const uint8_t* p = base + (i >> 1) * 4096 + (i & 1) * 512;
    const i32x4 lo = *(const i32x4*)(p + fw0), hi = *(const i32x4*)(p + (fw0 ^ 64u));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto frag_x = [&](const uint8_t* base, int j) {
    const uint8_t* p = base + j * 2048;
    const i32x4 lo = *(const i32x4*)(p + fx0), hi = *(const i32x4*)(p + (fx0 ^ 64u));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto scale_of = [&](uint32_t bits) {
    return E8 ? e8m0_value(bits) : __uint_as_float(bits);
  };

  const bool scales_w = w >= 4;
  HeadTile<E8> cur(a, t, tiles, scales_w);
  HeadTile<E8> next(a, t + step < t1 ? t + step : tiles, tiles, scales_w);
#pragma unroll
  for (int k = 0; k < 8; ++k) ask(cur, 0, k);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    put(0, k);
    ask(cur, 1, k);
  }
  const int nb = max(a.nb, 2);  // (a second block of zeros, so that two stages are this tile's)
  int buf = 0;
  for (;;) {
    f32x4 acc[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int b = 0; b < nb; ++b, buf ^= 1) {
      const uint8_t* fw = lds[buf][0] + wv * 128;
      const uint8_t* fx = lds[buf][1] + wn * 128;
      const bool over = b + 2 >= nb;  // stage g + 2 is the next tile's
      HeadTile<E8> from = cur;
      from.w = over ? next.w : cur.w;
      from.x = over ? next.x : cur.x;
      from.s = over ? next.s : cur.s;
      from.wbytes = over ? next.wbytes : cur.wbytes;
      from.xbytes = over ? next.xbytes : cur.xbytes;
      from.sbytes = over ? next.sbytes : cur.sbytes;
      const int fb = over ? b + 2 - nb : b + 2;
      __syncthreads();  // stage g is in LDS; the other half is free
      if (ODD && b == a.nb - 1) {
        // a thread per row cuts what follows H in the piece that holds the row's end
        // (as pieces pass through registers, it would cost registers that hold sums)
        const uint32_t row = (uint32_t)tid & 255u, at = ((uint32_t)a.H >> 4) & 7u;
        const uint32_t key = tid < 256 ? key_w(row) : key_x(row);
        u32x4* p = (u32x4*)(lds[buf][tid >> 8] + row * 128 + ((at ^ key) << 4));
        *p = keep16(*p, 0, (int)a.H & 15);
        __syncthreads();
      }
      const uint32_t hs = lsc[buf][kTileN + (w & 1)];
#pragma unroll
      for (int h = 0; h < 4; h += JH) {
        Frag<TO> bx[JH];
        i32x8 aw[PF];
        uint32_t ts[JH];
        float s[JH];
        f32x4 p[2][JH];
#pragma unroll
        for (int j = 0; j < JH; ++j) {
          bx[j] = Frag<TO>(frag_x(fx, h + j));
          ts[j] = lsc[buf][wn + 16 * (h + j) + lr];
        }
#pragma unroll
        for (int i = 0; i < PF - 1; ++i) aw[i] = frag_w(fw, i);
        if constexpr (!HW) {
#pragma unroll
          for (int j = 0; j < JH; ++j) s[j] = scale_of(ts[j]) * scale_of(hs);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < (HW ? 8 : 9); ++i) {
          if (i < 9 - PF) aw[(i + PF - 1) % PF] = frag_w(fw, i + PF - 1);
          const int k = h / JH * 8 + i - FIRST;
          if (i < 8 && k >= 0 && k < 8) {
            put(buf ^ 1, k);
            ask(from, fb, k);
          }
          if constexpr (HW) {
#pragma unroll
            for (int j = 0; j < JH; ++j)
              acc[i & 7][h + j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                  aw[i % PF], bx[j].v, acc[i & 7][h + j], 0, 0, 0, (int)hs, 0, (int)ts[j]);
          } else if constexpr (WIDE) {
            // (the registers hold one set of products)
            if (i < 8) {
              const Frag<TO> head(aw[i % PF]);
#pragma unroll
              for (int j = 0; j < JH; ++j) p[0][j] = mma128<TO>(head, bx[j]);
#pragma unroll
              for (int j = 0; j < JH; ++j) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  acc[i & 7][h + j][e] = fmaf(p[0][j][e], s[j], acc[i & 7][h + j][e]);
                asm volatile("" : "+v"(acc[i & 7][h + j]));
              }
            }
          } else {
            if (i < 8) {
#pragma unroll
              for (int j = 0; j < JH; ++j) p[i & 1][j] = mma128<TO>(Frag<TO>(aw[i % PF]), bx[j]);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (i > 0) {  // the products before are added meanwhile
#pragma unroll
              for (int j = 0; j < JH; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  acc[i - 1][h + j][e] = fmaf(p[(i - 1) & 1][j][e], s[j], acc[i - 1][h + j][e]);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t n = cur.n0 + wn + 16 * j + lr;
      if (n < a.N) {
        char* row = (char*)a.out + n * a.ldo * TO::BYTES;
#pragma unroll
        for (int i = 0; i < 8; i += 2)
          store8_logits<TO>(row, cur.v0 + wv + 16 * i + 8 * lk, a.V, acc[i][j], acc[i + 1][j]);
      }
    }
    t += step;
    if (t >= t1) break;
    cur = next;
    next = HeadTile<E8>(a, t + step < t1 ? t + step : tiles, tiles, scales_w);
  }
}

// Up to 128 tokens, or so few logits that their tiles leave CUs idle, the rows are
// streamed (for every 128 tokens again).  Streamed / tiled at H = 4,096, us:
//                              bf16 logits,           fp32 logits,
//   tokens x V                 fp32 scales  e8m0      fp32 scales
//   512 x 8,000    (4.1 M)      39 / 61      33 / 50     58 / 119
//   1,024 x 8,000  (8.2 M)      68 / 75      59 / 57    101 / 127
//   256 x 32,000   (8.2 M)      69 / 140     64 / 104   104 / 229
//   384 x 32,000   (12.3 M)    103 / 122     92 / 100   145 / 225
//   256 x 50,257   (12.9 M)    123 / 142    111 / 110   172 / 227
//   512 x 32,000   (16.4 M)    127 / 132    117 / 106   191 / 239
//   2,048 x 8,000  (16.4 M)    123 / 78     113 / 61    181 / 135
//   384 x 50,257   (19.3 M)    154 / 132    137 / 108   221 / 235
//   136 x 151,936  (20.7 M)    305 / 204    293 / 177   419 / 345
//   1,024 x 32,000 (32.8 M)    236 / 156    216 / 124   352 / 260
// and the same to either side at H = 512, 2,048 and 8,192.  One bound for all loses up to
// a seventh for bf16 logits (e8m0, 1,024 x 8,000 at H = 8,192), and for fp32 ones up to a third
// where 14 to 20 million are of few tokens (512 x 32,000 at H = 512: 36 / 49).
constexpr int64_t kFewLogits = 14000000;
template <class TO, bool E8>
hipError_t launch_head_t(HeadArgs a, hipStream_t stream) {
  if (a.N <= 128 || a.N * a.V <= kFewLogits) return launch_few<TO, E8>(a, stream);
  a.ntiles = (a.N + kTileN - 1) / kTileN;
  const int64_t tiles = (a.V + kTileV - 1) / kTileV * a.ntiles;
  const auto kernel = a.H % 16 != 0 ? k_head_tile<TO, E8, true> : k_head_tile<TO, E8, false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)min(tiles, (int64_t)kHeadCus)),
                     dim3(kTileThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize(const QuantArgs& a, int in_dt, bool e8m0, hipStream_t stream) {
  if (in_dt == BF16)
    return e8m0 ? launch_quantize_t<InBf16, true>(a, stream)
                : launch_quantize_t<InBf16, false>(a, stream);
  return e8m0 ? launch_quantize_t<InF32, true>(a, stream)
              : launch_quantize_t<InF32, false>(a, stream);
}

hipError_t launch_head(const HeadArgs& a, int out_dt, bool e8m0, hipStream_t stream) {
  if (out_dt == BF16)
    return e8m0 ? launch_head_t<OutBf16, true>(a, stream) : launch_head_t<OutBf16, false>(a, stream);
  return e8m0 ? launch_head_t<OutF32, true>(a, stream) : launch_head_t<OutF32, false>(a, stream);
}

}  // namespace opd
