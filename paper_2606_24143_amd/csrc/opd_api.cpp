// C-ABI entry points of libopd: argument validation, path selection, launch.
// Every argument check runs on the host before any HIP call, so argument
// errors are reported without touching the device.
#include <limits.h>
#include <stdint.h>

#include "../../include/opd.h"
#include "opd_internal.h"
#include "opd_model.h"

namespace {

using opd::Args;
using opd::Path;

// Below this many rows the split-vocabulary path runs (when it has a
// workspace): so few rows leave most of the 256 CUs idle, and splitting the
// rows over more workgroups outweighs the split path's second read of each
// row.  Measured on MI355X (16-sample MC, V = 151,936 bf16, inputs rotated
// so no step finds the last one's rows in the Infinity Cache), mean time per
// call, split against row path: N = 8: 9.8 against 22.7 us; 24: 13.9 against
// 23.3; 48: 17.9 against 23.6; 63: 20.1 against 23.9; more rows 128: 44.9
// against 31.3.  Dense: N = 63: 24.5 against 30.5.
constexpr int64_t kSplitMaxRows = 64;
// Workgroups the split path aims for below kSplitMaxRows: six to a CU, all of
// them resident at once (two or three rounds of shorter ones repeat the rows'
// merge and estimator in each).  Against 8,192 (64 chunks per row), V = 151,936:
// bf16 MC N = 48: 17.5 against 20.4 us; 63: 19.9 / 24.0; fp32 63: 24.5 / 30.4;
// dense bf16 63: 24.5 / 29.6; V = 60,000 48: 13.1 / 18.7.  512 and 1,024: 23.4
// and 22.2 us where 1,536 takes 19.6; 2,048: 23.5.
constexpr int64_t kSplitResidentGroups = 1536;
// Two kinds of calls keep 64 chunks.  Those that read more than the caches hold
// between the passes are bound by memory, where more and shorter workgroups
// leave less idle at the end: dense fp32 V = 300,000 N = 40 (96 MB): 45.3 against 47.2
// us, 63: 64.7 / 67.4; 250,000 56: 48.8 / 52.5; but 151,936 63 (77 MB): 37.3 / 36.5.  And
// up to 32 rows whose chunks are then four to five vectors per lane, of 2-byte
// logits or an estimator that writes without reading again: their 2,048 workgroups
// (eight to a CU) are all resident too, and 48 chunks would take six or seven
// vectors: bf16 MC V = 262,144 N = 32: 17.8 / 19.4, 300,000: 19.6 / 21.2; fp32 top-k with
// the log-partition 262,144: 19.4 / 20.8; but bf16 MC 400,000: 25.4 / 24.2.
constexpr int64_t kSplitResidentBytes = 78000000;
// The workspace's size, and the chunks of forced calls over more rows, come
// from this target and the largest chunk count.
constexpr int64_t kSplitTargetGroups = 8192;
constexpr int kSplitMaxChunks = 64;

constexpr uint32_t kKnownFlags =
    OPD_FLAG_SKIP_MASKED | OPD_FLAG_FORCE_ROWWISE | OPD_FLAG_FORCE_SPLITV;

bool valid_est(int32_t e) { return e >= OPD_FKL_TOPK && e <= OPD_RKL_TOPK_TRUNC; }
// renormalised top-k: only the k cached logits are needed
bool est_topk(int32_t e) { return e == OPD_FKL_TOPK || e == OPD_RKL_TOPK; }
bool est_trunc(int32_t e) { return e == OPD_FKL_TOPK_TRUNC || e == OPD_RKL_TOPK_TRUNC; }
// every estimator that reads the top-k cache (idx, k)
bool est_support(int32_t e) { return est_topk(e) || est_trunc(e); }
bool est_mc(int32_t e) {
  return e == OPD_RKL_MC1 || e == OPD_RKL_MC || (e >= OPD_RKL_MC_CLIP && e <= OPD_RKL_MC_NOIS);
}
bool est_clip(int32_t e) { return e == OPD_RKL_MC_CLIP || e == OPD_RKL_MC_OLD_CLIP; }

int mc_variant(int32_t e) {
  switch (e) {
    case OPD_RKL_MC_CLIP: return opd::MC_THETA_CLIP;
    case OPD_RKL_MC_OLD: return opd::MC_OLD;
    case OPD_RKL_MC_OLD_CLIP: return opd::MC_OLD_CLIP;
    case OPD_RKL_MC_NOIS: return opd::MC_NO_IS;
    case OPD_FKL_TOPK_TRUNC: return opd::TRUNC_FKL;
    case OPD_RKL_TOPK_TRUNC: return opd::TRUNC_RKL;
  }
  return opd::MC_THETA;
}

// The kernel family an estimator runs: the MC family and the truncated top-k
// KLs run the RKL_MC kernels (dense coefficient plus spikes).
int kernel_est(int32_t e) { return est_mc(e) || est_trunc(e) ? (int)opd::RKL_MC : (int)e; }
bool est_dense(int32_t e) { return e == OPD_FKL_DENSE || e == OPD_RKL_DENSE; }
int elt_bytes(int32_t dt) { return dt == OPD_BF16 ? 2 : 4; }
int elems_per_vec(int32_t) { return opd::kElemsPerVec; }

int check_shape(int64_t N, int64_t V, int64_t ld) {
  if (N < 0 || N > INT32_MAX) return OPD_ERR_SHAPE;
  if (V < 2 || V > INT32_MAX) return OPD_ERR_SHAPE;
  if (ld < V) return OPD_ERR_SHAPE;
  return OPD_OK;
}

int check_support(int32_t est, int64_t V, int32_t k, int32_t M) {
  if (est_support(est)) {
    const int64_t kmax = V < OPD_K_MAX ? V : OPD_K_MAX;
    if (k < 1 || k > kmax) return OPD_ERR_SUPPORT;
  } else if (est_mc(est)) {
    if (M < 1 || M > OPD_K_MAX) return OPD_ERR_SUPPORT;
    if (est == OPD_RKL_MC1 && M != 1) return OPD_ERR_SUPPORT;
  }
  return OPD_OK;
}

int check_flags(uint32_t flags) {
  if (flags & ~kKnownFlags) return OPD_ERR_FLAGS;
  if ((flags & OPD_FLAG_FORCE_ROWWISE) && (flags & OPD_FLAG_FORCE_SPLITV)) return OPD_ERR_FLAGS;
  return OPD_OK;
}

struct Plan {
  bool split;
  int P;
  int64_t chunk_vec;
  size_t ws_bytes;
};

// The split-path layout for N rows of nvec vectors: enough chunks for about
// kSplitTargetGroups workgroups (kSplitResidentGroups below kSplitMaxRows rows,
// but see there), each chunk at least one vector per lane.  The workspace is
// sized for the former, so a size that serves some rows serves fewer.
Plan split_plan(int64_t N, int64_t nvec, int32_t dtype, int32_t est) {
  const int vec_bytes = elems_per_vec(dtype) * elt_bytes(dtype) * (est_dense(est) ? 2 : 1);
  Plan p{true, 1, nvec, 0};
  int64_t P = (kSplitTargetGroups + N - 1) / N;
  const int64_t by_width = nvec / opd::kSplitThreads;
  if (P > by_width) P = by_width;
  if (P > kSplitMaxChunks) P = kSplitMaxChunks;
  if (P < 1) P = 1;
  p.ws_bytes = (size_t)N * (size_t)P * opd::kPartialFloats * sizeof(float);
  const int64_t resident = (kSplitResidentGroups + N - 1) / N;
  const int64_t one = kSplitMaxChunks * opd::kSplitThreads;  // vectors of one per lane
  const bool many = N * nvec * vec_bytes > kSplitResidentBytes ||
                    (N <= kSplitMaxRows / 2 && nvec >= 4 * one && nvec <= 5 * one &&
                     (est_topk(est) || (dtype == OPD_BF16 && !est_dense(est))));
  if (N < kSplitMaxRows && !many && P > resident) P = resident;
  p.P = (int)P;
  p.chunk_vec = (nvec + P - 1) / P;
  return p;
}

bool split_wanted(int64_t N, uint32_t flags) {
  if (flags & OPD_FLAG_FORCE_SPLITV) return true;
  if (flags & OPD_FLAG_FORCE_ROWWISE) return false;
  return N < kSplitMaxRows;
}

// Below kSplitMaxRows rows, those that stay whole: the register-resident
// kernel's classes that share a CU, one launch of one read, where its longer
// chain (a lane's slots, then the cache entries, which one wave handles while the
// others wait) is no longer than the split path's two launches.
// Measured, split against row path, Monte-Carlo with K draws: K = 1 bf16 V = 16,384
// N = 8: 7.3 / 7.0 us, 24,576 8: 7.4 / 7.6; K = 16 bf16 2,000 8: 9.6 / 6.1, 12,000 8: 9.0 /
// 8.2, 16,384 8: 8.0 / 8.5 and 63: 10.8 / 9.5, 32,768 8: 8.1 / 9.7 and 24: 9.7 / 9.6; fp32
// 16,384 8: 7.9 / 6.9; K = 32 bf16 4,096 8: 8.4 / 8.0, 8,192 63: 9.5 / 10.3, 32,768 8: 8.4 /
// 10.7 and 63: 14.2 / 11.3; fp32 8,192 8: 8.3 / 9.0, 16,384 24: 8.9 / 8.7; K = 48 bf16 2,000
// (one chunk) 8: 10.7 / 9.5, 4,096 8: 8.8 / 9.8, 32,768 63: 14.9 / 13.1; K = 64 bf16 4,096 8:
// 9.1 / 11.2, 24,576 63: 13.7 / 14.5; K = 128 bf16 8,192 8: 13.3 / 21.6.  The renormalised
// top-k with the log-partition, K = 32: fp32 2,000 8: 10.3 / 8.8, 8,192 8: 8.6 / 9.2, 16,384
// 63: 11.9 / 11.2; bf16 16,384 8: 8.7 / 10.1.  Wider rows, K = 16, 60,000 8: 9.5 / 11.7;
// dense rows have no such class: V = 32,000 63: 13.0 / 16.3.
bool whole_rows(int64_t N, int64_t nvec, int32_t dtype, int32_t est, int K, uint32_t flags) {
  if ((flags & OPD_FLAG_FORCE_SPLITV) || est_dense(est)) return false;
  const int64_t slots = opd::slots_small(dtype);
  if (nvec > slots * (opd::kRowThreads / 2)) return false;
  const bool f32 = dtype == OPD_F32;
  const bool wide = nvec > slots * (opd::kRowThreads / 4);  // 512 lanes to a row
  if (est_topk(est)) return f32 && K <= 32 && (nvec <= 512 || (wide && N >= 56));
  if (K <= 8) return f32 || nvec <= 4096 || N >= 24;
  if (K <= 16) return f32 || nvec <= 3072 || N >= (wide ? 24 : 32);
  if (K <= 32) return nvec <= 1024 || (wide && (f32 || N >= 40));
  return K <= 48 && ((nvec > 256 && nvec <= 512) || (wide && N >= 56));
}

int64_t nvec_of(int64_t V, int32_t dt) {
  const int64_t epv = elems_per_vec(dt);
  return (V + epv - 1) / epv;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

// A HIP grid holds fewer than 2^32 work-items: calls with more rows than one
// grid takes run as consecutive launches over row chunks.
constexpr int64_t kMaxGridLanes = 0xFFFFFFFFll;

// The arguments of rows [r0, r0 + n) of a loss call: every row-indexed
// pointer moves to row r0.
Args loss_rows(const Args& a, int64_t r0, int64_t n, int in_bytes, int out_bytes) {
  Args b = a;
  b.N = n;
  b.logits = (const char*)a.logits + r0 * a.ld * in_bytes;
  if (a.teacher) b.teacher = (const char*)a.teacher + r0 * a.ld * in_bytes;
  b.dlogits = (char*)a.dlogits + r0 * a.ld * out_bytes;
  if (a.ids) b.ids = a.ids + r0 * a.K;
  if (a.tau) b.tau = a.tau + r0 * a.K;
  if (a.beta) b.beta = a.beta + r0 * a.K;
  if (a.mask) b.mask = a.mask + r0;
  b.loss = a.loss + r0;
  if (a.lse_out) b.lse_out = a.lse_out + r0;
  if (a.gathered_out) b.gathered_out = a.gathered_out + r0 * a.K;
  if (a.coverage_out) b.coverage_out = a.coverage_out + 2 * r0;
  if (a.ws) b.ws = a.ws + r0 * a.P * opd::kPartialFloats;
  return b;
}

// The same for a cache-building call.
opd::CacheArgs cache_rows(const opd::CacheArgs& a, int64_t r0, int64_t n, int in_bytes) {
  opd::CacheArgs b = a;
  b.N = n;
  b.logits = (const char*)a.logits + r0 * a.ld * in_bytes;
  if (a.u) b.u = a.u + r0 * a.K;
  if (a.ids) b.ids = a.ids + r0 * a.K;
  if (a.mask) b.mask = a.mask + r0;
  if (a.ids_out) b.ids_out = a.ids_out + r0 * a.K;
  if (a.logp) b.logp = a.logp + r0 * a.K;
  if (a.lse_out) b.lse_out = a.lse_out + r0;
  return b;
}

// Launches a cache-building op over row chunks that each fit one grid
// (at most 1024 lanes per row).
hipError_t launch_cache_chunks(const opd::CacheArgs& a, opd::CacheOp op, int32_t dtype,
                               bool resident, hipStream_t s) {
  const int64_t max_rows = kMaxGridLanes / opd::kRowThreads;
  for (int64_t r0 = 0; r0 < a.N; r0 += max_rows) {
    const int64_t n = a.N - r0 < max_rows ? a.N - r0 : max_rows;
    const hipError_t e = opd::launch_cache(cache_rows(a, r0, n, elt_bytes(dtype)), op, dtype,
                                           resident, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Arguments shared by the cache-building entry points.
int check_row_call(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t ld, int32_t K,
                   int64_t kmax) {
  if (dtype != OPD_F32 && dtype != OPD_BF16) return OPD_ERR_DTYPE;
  if (int rc = check_shape(N, V, ld)) return rc;
  if (K < 1 || K > kmax) return OPD_ERR_SUPPORT;
  if (N > 0 && (!aligned16(logits) || (ld * elt_bytes(dtype)) % 16 != 0)) return OPD_ERR_ALIGN;
  return OPD_OK;
}

opd::CacheArgs row_args(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t ld,
                        int32_t K, const uint8_t* mask, float* logp, float* lse_out) {
  opd::CacheArgs a{};
  a.logits = logits;
  a.N = N;
  a.V = V;
  a.ld = ld;
  a.nvec = nvec_of(V, dtype);
  a.tail = (int)(V - (a.nvec - 1) * elems_per_vec(dtype));
  a.K = K;
  a.mask = mask;
  a.logp = logp;
  a.lse_out = lse_out;
  return a;
}

// A row that fits the registers of one workgroup is read once.
bool row_fits(int64_t nvec, int32_t dtype) {
  return nvec <= (int64_t)opd::slots_large(dtype) * opd::kRowThreads;
}

// Arguments shared by the blockwise calls.
// (the head's kernels address the rows of a tile within 2 GiB, count tiles of 2^16
// logits in 32 bits, and have four work-items to a row of the head)
constexpr int64_t kMaxHidden = (int64_t)1 << 22, kMaxHeadRows = (int64_t)1 << 29;
constexpr int64_t kMaxLogits = (int64_t)1 << 46;
int check_blocks(int64_t N, int64_t H, int32_t scale_type) {
  if (scale_type != OPD_SCALE_F32 && scale_type != OPD_SCALE_E8M0) return OPD_ERR_DTYPE;
  if (N < 0 || N > INT32_MAX || H < 1 || H > kMaxHidden) return OPD_ERR_SHAPE;
  return OPD_OK;
}

int check_verify(int32_t dtype, int64_t B, int32_t D, int64_t V, int64_t ld, int64_t draft_ld) {
  if (dtype != OPD_F32 && dtype != OPD_BF16) return OPD_ERR_DTYPE;
  if (D < 1 || D > OPD_K_MAX) return OPD_ERR_SUPPORT;
  if (int rc = check_shape(B, V, ld)) return rc;
  if (B * (D + 1) > INT32_MAX || draft_ld < V) return OPD_ERR_SHAPE;
  return OPD_OK;
}

// How the rows of a verification are split.
struct VerifyPlan {
  int parts, draw_parts, nchunk, chunk_steps, round;
  uint32_t part_groups;
  bool table;
  size_t ws_bytes;
};
VerifyPlan verify_plan(int64_t B, int32_t D, int64_t V, int32_t dtype, bool draft) {
  VerifyPlan p{};
  const int64_t groups = (V + 7) / 8;
  const int64_t steps = (groups + 63) / 64;  // of 512 elements
  // a row's parts, one to a wavefront, of whole tiles of 256 groups: at most (k_verify_rows
  // takes as few as fill the GPU, or these where there are too many rows to count)
  const int64_t tiles = (groups + 255) / 256;
  int64_t parts = 16384 / B;
  if (parts > tiles) parts = tiles;
  if (parts > 64) parts = 64;
  if (parts < 4) parts = tiles < 4 ? tiles : 4;
  const int64_t per = (tiles + parts - 1) / parts;
  p.parts = (int)((tiles + per - 1) / per);
  p.part_groups = (uint32_t)(per * 256);
  p.chunk_steps = (int)((steps + opd::kVerMaxChunks - 1) / opd::kVerMaxChunks);
  p.nchunk = (int)((steps + p.chunk_steps - 1) / p.chunk_steps);
  // the draw's parts, one to a workgroup: of 4,096 elements at least, and as many as
  // all have a workgroup at once, since a few left over take a turn of their own.  Rounded
  // down / up, us: V = 151,936, 100 sequences 93 / 105, 257 178 / 187, 300 196 / 205; V =
  // 32,000, 200 69 / 75, 300 75 / 84; fp32 V = 50,257, 100 50 / 57.
  int64_t k = opd::kVerGroups / B;
  if (k > groups / 512) k = groups / 512;
  p.draw_parts = k < 1 ? 1 : (int)k;
  // Terms of bf16 rows from a table, which costs each workgroup some 3 us: D = 4, with /
  // without it, us: V = 151,936, B = 8 47 / 46, 16 51 / 50, 26 52 / 59, 40 57 / 71;
  // V = 32,000, B = 32 36 / 35, 64 39 / 42, 128 51 / 61.
  p.table = B * V >= 2000000;
  // The first round's positions: some 32 M elements (fp32 rows, bound by arithmetic, take as
  // long as bf16 ones).  Every round costs about 12 us besides (a launch, the table,
  // the tests at its end), so small ones do not pay; later ones have twice the
  // positions, as fewer sequences are left.  First rounds of 2 / 4 / 6 positions, us: 64
  // sequences of 5 drafts, bf16 V = 151,936 80 / 86 / 80; of 2 / 3 / 6: 256 of 8 drafts,
  // fp32 V = 50,257 100 / 96 / 118.
  constexpr int64_t kRoundElements = (int64_t)32 << 20;
  const int64_t round = kRoundElements / ((draft ? 2 : 1) * B * V) + 1;
  p.round = (int)(round < D + 1 ? round : D + 1);
  const size_t rows = (size_t)B * (size_t)(2 * D + 1);
  p.ws_bytes = rows * 16 * (1 + (size_t)p.parts) +
               (p.draw_parts > 1 ? (size_t)B * p.nchunk * 8 : 0) +
               (size_t)B * (2 * (size_t)(D + 1) + 2) * 4;
  return p;
}

// Arguments shared by the calls on rows of an embedding table.
int check_embed(int32_t dtype, int32_t other, int64_t N, int64_t V, int64_t H) {
  if ((dtype != OPD_F32 && dtype != OPD_BF16) || (other != OPD_F32 && other != OPD_BF16))
    return OPD_ERR_DTYPE;
  if (N < 0 || N > INT32_MAX || V < 1 || V > INT32_MAX || H < 1 || H > kMaxHidden)
    return OPD_ERR_SHAPE;
  return OPD_OK;
}
bool rows_aligned(const void* p, int64_t ld, int32_t dtype) {
  return aligned16(p) && (ld * elt_bytes(dtype)) % 16 == 0;
}
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// Workspace of opd_embed_grads: first places, sorted tokens, sums of tiles.
struct EmbedLayout {
  size_t perm, partial, total;
  int64_t hp;
};
// Few tokens are looked for by each entry's wavefronts themselves: 64, which they load at
// once, or up to 256 where there are few wavefronts.  256 tokens: 27.1 us unsorted and 33.1
// sorted for 32,000 by 1,000 fp32, 411 and 362 for 151,936 by 4,096; 64: 26.2 and 33.2, 365 and
// 360.
bool embed_unsorted(int64_t N, int64_t V, int64_t H) {
  return N <= 64 || (N <= 256 && V * ((H + 255) / 256) <= (1 << 18));
}
EmbedLayout embed_layout(int64_t N, int64_t V, int64_t H) {
  EmbedLayout l{};
  l.hp = (H + 7) / 8 * 8;
  if (embed_unsorted(N, V, H)) return l;
  l.perm = up256((size_t)(V + 1) * 4);
  l.partial = l.perm + up256((size_t)N * 4);
  l.total = l.partial + up256((size_t)((N + opd::kEmbTile - 1) / opd::kEmbTile) * 2 * (size_t)l.hp * 4);
  return l;
}
// Entries to a workgroup that sorts: about a workgroup to each CU, up to kEmbKeys entries.  The
// gradient of 4,096 tokens of 64 columns: 16.3 us for 32,000 entries (64 to a workgroup 20.1,
// 512 17.6), 14.6 for 2,000 (512 15.8); of 16,384 for 151,936 43.5 (64 90.7).
int embed_keys(int64_t V) {
  int keys = 64;
  while (keys < opd::kEmbKeys && (int64_t)keys * 300 < V) keys *= 2;
  return keys;
}

// Arguments shared by the calls on adapters.
constexpr int64_t kMaxAdaptTokens = (int64_t)1 << 24;
int check_adapters(int32_t dtype, int32_t y_dtype, int64_t N, int64_t H, int64_t O, int32_t G,
                   int32_t r) {
  if (dtype != OPD_F32 && dtype != OPD_BF16) return OPD_ERR_DTYPE;
  if (y_dtype != OPD_F32 && y_dtype != dtype) return OPD_ERR_DTYPE;
  if (N < 0 || N > kMaxAdaptTokens || H < 1 || H > kMaxHidden || O < 1 || O > kMaxHidden)
    return OPD_ERR_SHAPE;
  if (G < 1 || G > OPD_ADAPTERS_MAX || r < 1 || r > OPD_RANK_MAX) return OPD_ERR_SUPPORT;
  return OPD_OK;
}
// Workspace of the calls on adapters, and how their products are split.
struct AdaptLayout {
  int64_t max_tiles, ldt;
  int64_t span_x, span_y;      // of the long axes, parts
  int splits_x, splits_y;
  int outer;                   // parts of an adapter's tokens
  size_t start, tiles, t, u, part_x, part_y, total;
};
// Parts of a long axis of D columns: about 256 workgroups of 16 tokens, each
// with 1,024 columns at least.  4,096 columns, the whole call: 1 token 6.9 us (undivided 8.3),
// 64 of 32 adapters 9.6 (9.9); 2,048 of 4 20.6 undivided, 23.3 in four parts.
void split_axis(int64_t groups, int64_t D, int64_t* span, int* splits) {
  int64_t s = 256 / groups, most = D / 1024;
  if (s > most) s = most;
  if (s < 1) s = 1;
  *span = ((D + s - 1) / s + 511) / 512 * 512;
  *splits = (int)((D + *span - 1) / *span);
}
AdaptLayout adapt_layout(int64_t N, int64_t H, int64_t O, int32_t G, int32_t r, int32_t dtype,
                         int32_t y_dtype, bool backward) {
  AdaptLayout l{};
  const int64_t keys = (int64_t)G + 2 < N ? (int64_t)G + 2 : N;
  l.max_tiles = N / opd::kAdTile + keys;
  l.ldt = (r + 3) / 4 * 4;
  const int64_t groups = N / 16 + (keys + 1) / 2 + 1;
  split_axis(groups, H, &l.span_x, &l.splits_x);
  split_axis(groups, O, &l.span_y, &l.splits_y);
  size_t at = up256((size_t)N * 4);  // perm
  l.start = at;
  at += up256((size_t)(G + 3) * 4);
  l.tiles = at;
  at += up256((size_t)l.max_tiles * sizeof(opd::AdTile));
  l.t = at;
  at += up256((size_t)l.splits_x * N * l.ldt * 4);
  l.u = at;
  if (backward) {
    at += up256((size_t)l.splits_y * N * l.ldt * 4);
    l.part_x = at;
    const int64_t used = G < N ? G : N;
    // parts of an adapter's tokens, of which a workgroup's waves take 256 at once: four
    // workgroups to a CU, both sums together (8,192 tokens of 4 adapters by 4,096 columns: 4
    // parts 30.2 us and 5 for their sums, 2 35.6 and 5, 8 35.5 and 5, undivided 39.9)
    const int64_t chunks = (H + (dtype == OPD_BF16 ? 127 : 63)) / (dtype == OPD_BF16 ? 128 : 64) +
                           (O + (y_dtype == OPD_BF16 ? 127 : 63)) / (y_dtype == OPD_BF16 ? 128 : 64);
    int64_t s = 1024 / (chunks * (used > 0 ? used : 1));
    if (s > N / 512) s = N / 512;
    l.outer = (int)(s < 1 ? 1 : s);
    const size_t gr = (size_t)l.outer * (size_t)G * (size_t)r * 4;
    l.part_y = l.part_x + up256(l.outer > 1 ? gr * (size_t)((H + 3) / 4 * 4) : 0);
    at = l.part_y + up256(l.outer > 1 ? gr * (size_t)((O + 3) / 4 * 4) : 0);
  }
  l.total = at;
  return l;
}
// (a launch has fewer than 2^32 work-items)
bool adapt_fits(const AdaptLayout& l, int64_t D, int32_t G, bool backward) {
  const int64_t chunks = (D + 63) / 64, splits = l.splits_x + l.splits_y;
  if (l.max_tiles * 4 * 512 * splits > kMaxGridLanes) return false;
  if (!backward) return true;
  return (int64_t)G * l.outer * 2 * chunks * 2 * 512 <= kMaxGridLanes;
}

// How rows of logits are cut for the selection of beams.
int check_beams(int32_t dtype, int64_t B, int32_t W, int64_t V, int64_t ld) {
  if (dtype != OPD_F32 && dtype != OPD_BF16) return OPD_ERR_DTYPE;
  if (W < 1 || W > OPD_BEAM_MAX) return OPD_ERR_SUPPORT;
  if (int rc = check_shape(B, V, ld)) return rc;
  if (B > INT32_MAX / opd::kBeamMax / 16) return OPD_ERR_SHAPE;
  return OPD_OK;
}
struct BeamPlan {
  int slots;
  int64_t parts;
  size_t cands, total;
};
// Parts of 8 vectors of 16 bytes a lane; fewer where that makes fewer than 1,024 workgroups, as
// long as a group's parts are no more than its merge takes at once.  bf16, the call on the
// GPU: 4 rows of 32,000 10.3 us with 1 vector (8: 11.1), 4 of 151,936 11.2 with 4
// (1: 18.0, 8: 11.6), 32 of 151,936 14.1 with 8 (1: 46.9).
BeamPlan beam_plan(int64_t B, int32_t W, int64_t V, int32_t dtype) {
  constexpr int64_t at_once = 128;
  const int64_t rows = B * W;
  BeamPlan p{8, 0, 0, 0};
  const auto parts = [&](int slots) {
    const int64_t part = 256 * (16 / elt_bytes(dtype)) * (int64_t)slots;
    return (V + part - 1) / part;
  };
  while (p.slots > 1 && rows * parts(p.slots) < 1024 && W * parts(p.slots / 2) <= at_once)
    p.slots /= 2;
  p.parts = parts(p.slots);
  p.cands = up256((size_t)rows * (size_t)p.parts * sizeof(opd::BeamRec));
  p.total = p.cands + (size_t)rows * (size_t)p.parts * opd::kBeamMax * 8;
  return p;
}

// Workspace of opd_mc_diagnostics: regions in order, each 256-byte aligned.
struct DiagLayout {
  size_t rho, x, psum, seq, parts, hist, total;
  int64_t nseq, pieces;
  int seq_groups;
};

DiagLayout diag_layout(int64_t N, int32_t M, int32_t n_groups, int64_t seq_len) {
  DiagLayout l{};
  auto take = [&](size_t bytes) {
    const size_t at = l.total;
    l.total += (bytes + 255) & ~(size_t)255;
    return at;
  };
  const bool seq = seq_len > 0 && n_groups > 0;
  l.nseq = seq ? (N + seq_len - 1) / seq_len : 0;
  l.pieces = seq ? opd::diag_pieces(N, seq_len) : 0;
  l.rho = take((size_t)N * M * 4);
  l.x = seq ? take((size_t)N * M * 4) : 0;
  l.psum = l.pieces > 0 ? take((size_t)(l.nseq * l.pieces) * (M + 1) * 8) : 0;
  l.seq_groups = seq ? opd::diag_seq_groups(l.nseq, M, n_groups) : 0;
  l.seq = seq ? take((size_t)l.seq_groups * (opd::kDiagMaxGroups + 1) * 8) : 0;
  l.parts = take((size_t)opd::diag_parts(N) * (3 + opd::kDiagMaxGroups) * 8);
  l.hist = take((size_t)opd::kDiagHistWords * 4);
  return l;
}

// The diagnostics reduce over the whole batch in one grid of 64 lanes per
// token, so one call takes fewer than 2^32 / 64 tokens.
constexpr int64_t kDiagMaxRows = 0xFFFFFFFFll / 64;

int check_diag(int64_t N, int32_t M, float q, float clip_eps, const int32_t* groups,
               int32_t n_groups, int64_t seq_len) {
  if (N < 0 || N > kDiagMaxRows) return OPD_ERR_SHAPE;
  if (M < 1 || M > OPD_K_MAX) return OPD_ERR_SUPPORT;
  if (!(q > 0.0f && q <= 1.0f) || !(clip_eps >= 0.0f && clip_eps <= 3.0e38f)) return OPD_ERR_PARAM;
  if (n_groups < 0 || n_groups > opd::kDiagMaxGroups || seq_len < 0) return OPD_ERR_PARAM;
  if (n_groups > 0 && !groups) return OPD_ERR_NULL;
  for (int k = 0; k < n_groups; ++k)
    if (groups[k] < 1 || M % groups[k] != 0 || M / groups[k] < 2) return OPD_ERR_PARAM;
  return OPD_OK;
}

}  // namespace

extern "C" {

int opd_version(void) { return OPD_VERSION; }

const char* opd_status_string(int status) {
  switch (status) {
    case OPD_OK: return "ok";
    case OPD_ERR_NULL: return "a required pointer is NULL";
    case OPD_ERR_SHAPE: return "invalid shape (N, V or ld)";
    case OPD_ERR_SUPPORT: return "support size k or sample count M out of range";
    case OPD_ERR_DTYPE: return "unknown dtype";
    case OPD_ERR_ALIGN: return "pointer or row stride not 16-byte aligned";
    case OPD_ERR_WORKSPACE: return "workspace missing or too small for the split path";
    case OPD_ERR_ESTIMATOR: return "unknown estimator";
    case OPD_ERR_FLAGS: return "unknown or contradictory flags";
    case OPD_ERR_HIP: return "HIP runtime error";
    case OPD_ERR_PARAM: return "invalid scalar option or output (clip_eps, coverage_out, block_rows)";
    case OPD_ERR_SCRATCH:
      return "the call needs more scratch than the no-allocation entry point holds";
  }
  return "unknown status";
}

size_t opd_workspace_bytes(int64_t N, int64_t V, int32_t dtype, int32_t estimator, int32_t k,
                           int32_t M, uint32_t flags) {
  if (!valid_est(estimator) || (dtype != OPD_F32 && dtype != OPD_BF16)) return 0;
  if (check_shape(N, V, V) != OPD_OK || N == 0) return 0;
  if (check_support(estimator, V, k, M) != OPD_OK || check_flags(flags) != OPD_OK) return 0;
  if (!split_wanted(N, flags)) return 0;
  return split_plan(N, nvec_of(V, dtype), dtype, estimator).ws_bytes;
}

int opd_loss_fwd_bwd(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t ld,
                     const opd_cache* cache, int32_t estimator, int32_t k, int32_t M,
                     const uint8_t* mask, const opd_opts* opts, float* loss, void* dlogits,
                     float* lse_out, float* gathered_out, float* coverage_out, void* workspace,
                     size_t workspace_bytes, void* stream) {
  return opd::loss_call(logits, dtype, N, V, ld, cache, estimator, k, M, mask, opts, loss, dlogits,
                        lse_out, gathered_out, coverage_out, workspace, workspace_bytes, nullptr,
                        0, stream);
}

}  // extern "C"

namespace opd {

int loss_call(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t ld,
              const opd_cache* cache, int32_t estimator, int32_t k, int32_t M,
              const uint8_t* mask, const opd_opts* opts, float* loss, void* dlogits,
              float* lse_out, float* gathered_out, float* coverage_out, void* workspace,
              size_t workspace_bytes, ScratchFn scratch, size_t scratch_bytes, void* stream) {
  if (!valid_est(estimator)) return OPD_ERR_ESTIMATOR;
  const opd_opts o = opts ? *opts : opd_opts{1.0f, OPD_F32, 0u, 0.2f};
  if (dtype != OPD_F32 && dtype != OPD_BF16) return OPD_ERR_DTYPE;
  if (o.dlogits_dtype != OPD_F32 && o.dlogits_dtype != OPD_BF16) return OPD_ERR_DTYPE;
  if (int rc = check_flags(o.flags)) return rc;
  if (int rc = check_shape(N, V, ld)) return rc;
  if (int rc = check_support(estimator, V, k, M)) return rc;
  if (est_clip(estimator) && !(o.clip_eps > 0.0f && o.clip_eps <= 3.0e38f)) return OPD_ERR_PARAM;
  // support coverage exists only for the estimators that read a support
  if (coverage_out && !est_support(estimator)) return OPD_ERR_PARAM;
  if (N == 0) return OPD_OK;

  if (!logits || !cache || !loss || !dlogits) return OPD_ERR_NULL;
  const int32_t* ids = nullptr;
  int K = 0;
  if (est_support(estimator)) {
    if (!cache->idx || !cache->teacher_logp) return OPD_ERR_NULL;
    ids = cache->idx;
    K = k;
  } else if (est_mc(estimator)) {
    if (!cache->sampled_ids || !cache->teacher_logp) return OPD_ERR_NULL;
    if (estimator != OPD_RKL_MC_NOIS && !cache->behav_logp) return OPD_ERR_NULL;
    ids = cache->sampled_ids;
    K = M;
  } else {
    if (!cache->teacher_logits) return OPD_ERR_NULL;
  }

  if (!aligned16(logits) || !aligned16(dlogits)) return OPD_ERR_ALIGN;
  if (est_dense(estimator) && !aligned16(cache->teacher_logits)) return OPD_ERR_ALIGN;
  if ((ld * elt_bytes(dtype)) % 16 != 0) return OPD_ERR_ALIGN;
  if ((ld * elt_bytes(o.dlogits_dtype)) % 16 != 0) return OPD_ERR_ALIGN;

  const int64_t nvec = nvec_of(V, dtype);
  const int epv = elems_per_vec(dtype);
  const int tail = (int)(V - (nvec - 1) * epv);

  Plan plan{false, 1, nvec, 0};
  if (split_wanted(N, o.flags) && !whole_rows(N, nvec, dtype, estimator, K, o.flags)) {
    const Plan sp = split_plan(N, nvec, dtype, estimator);
    if (scratch) {
      // the no-allocation entry point: the library's static scratch array,
      // looked up only now that every argument has been checked
      if (sp.ws_bytes <= scratch_bytes) {
        workspace = scratch();
        if (!workspace) return OPD_ERR_HIP;
        plan = sp;
      } else if (o.flags & OPD_FLAG_FORCE_SPLITV) {
        return OPD_ERR_SCRATCH;
      }
    } else if (workspace && workspace_bytes >= sp.ws_bytes && aligned16(workspace)) {
      plan = sp;
    } else if (o.flags & OPD_FLAG_FORCE_SPLITV) {
      return OPD_ERR_WORKSPACE;
    }
  }

  Args a{};
  a.logits = logits;
  a.teacher = est_dense(estimator) ? cache->teacher_logits : nullptr;
  a.N = N;
  a.V = V;
  a.ld = ld;
  a.nvec = nvec;
  a.tail = tail;
  a.ids = ids;
  a.tau = est_dense(estimator) ? nullptr : cache->teacher_logp;
  a.beta = est_mc(estimator) && estimator != OPD_RKL_MC_NOIS ? cache->behav_logp : nullptr;
  a.K = K;
  a.mc_variant = mc_variant(estimator);
  a.clip_eps = o.clip_eps;
  a.mask = mask;
  a.gamma = o.grad_scale;
  a.skip_masked = (o.flags & OPD_FLAG_SKIP_MASKED) ? 1 : 0;
  a.loss = loss;
  a.dlogits = dlogits;
  a.lse_out = lse_out;
  a.gathered_out = est_dense(estimator) ? nullptr : gathered_out;
  a.coverage_out = coverage_out;
  a.ws = (float*)workspace;
  a.P = plan.P;
  a.chunk_vec = plan.chunk_vec;

  // The renormalised top-k estimators need the row itself only for lse_out
  // and the student's support coverage (both need L).
  const bool read_row = !est_topk(estimator) || lse_out != nullptr || coverage_out != nullptr;
  Path path = Path::RowStream;
  // register-resident rows (a partial last vector takes the kernels' TAIL
  // variant)
  if (nvec <= (int64_t)opd::slots_small(dtype) * opd::kRowThreads)
    path = Path::RowResidentSmall;
  else if (nvec <= (int64_t)opd::slots_large(dtype) * opd::kRowThreads)
    path = Path::RowResidentLarge;
  // rows per launch: the split grid has P workgroups of kSplitThreads lanes
  // per row, the others at most kRowThreads lanes per row (the top-k zero
  // fill chunks its own grid)
  const int64_t lanes_per_row =
      read_row && plan.split ? (int64_t)plan.P * opd::kSplitThreads : (int64_t)opd::kRowThreads;
  const int64_t max_rows = kMaxGridLanes / lanes_per_row;
  hipStream_t s = (hipStream_t)stream;
  hipError_t err = hipSuccess;
  for (int64_t r0 = 0; r0 < N && err == hipSuccess; r0 += max_rows) {
    const int64_t n = N - r0 < max_rows ? N - r0 : max_rows;
    const Args b = loss_rows(a, r0, n, elt_bytes(dtype), elt_bytes(o.dlogits_dtype));
    if (!read_row)
      err = opd::launch_topk_sparse(b, kernel_est(estimator), dtype, o.dlogits_dtype, s);
    else if (plan.split)
      err = opd::launch_split(b, kernel_est(estimator), dtype, o.dlogits_dtype, read_row, s);
    else
      err = opd::launch_rowwise(b, kernel_est(estimator), dtype, o.dlogits_dtype, path, read_row,
                                s);
  }
  return err == hipSuccess ? OPD_OK : OPD_ERR_HIP;
}

}  // namespace opd

extern "C" {

int opd_validate_cache(const opd_cache* cache, int32_t estimator, int64_t N, int64_t V,
                       int32_t k, int32_t M, int32_t* violations, void* stream) {
  if (!valid_est(estimator)) return OPD_ERR_ESTIMATOR;
  if (int rc = check_shape(N, V, V)) return rc;
  if (int rc = check_support(estimator, V, k, M)) return rc;
  if (est_dense(estimator) || N == 0) return OPD_OK;
  if (!cache || !violations) return OPD_ERR_NULL;
  const bool topk = est_support(estimator);
  const bool uses_beta = !topk && estimator != OPD_RKL_MC_NOIS;
  const int32_t* ids = topk ? cache->idx : cache->sampled_ids;
  if (!ids || !cache->teacher_logp || (uses_beta && !cache->behav_logp)) return OPD_ERR_NULL;
  const hipError_t err =
      opd::launch_validate(ids, cache->teacher_logp, uses_beta ? cache->behav_logp : nullptr, N,
                           V, topk ? k : M, topk ? 1 : 0, violations, (hipStream_t)stream);
  return err == hipSuccess ? OPD_OK : OPD_ERR_HIP;
}

int opd_sample_actions(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t ld,
                       int32_t M, const float* uniforms, const uint8_t* mask, int32_t* sampled_ids,
                       float* logp, float* lse_out, void* stream) {
  if (int rc = check_row_call(logits, dtype, N, V, ld, M, OPD_K_MAX)) return rc;
  if (N == 0) return OPD_OK;
  if (!logits || !uniforms || !sampled_ids) return OPD_ERR_NULL;
  opd::CacheArgs a = row_args(logits, dtype, N, V, ld, M, mask, logp, lse_out);
  a.u = uniforms;
  a.ids_out = sampled_ids;
  const hipError_t err = launch_cache_chunks(a, opd::CacheOp::Sample, dtype, row_fits(a.nvec, dtype),
                                           (hipStream_t)stream);
  return err == hipSuccess ? OPD_OK : OPD_ERR_HIP;
}

int opd_topk_support(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t ld, int32_t k,
                     const uint8_t* mask, int32_t* idx, float* logp, float* lse_out,
                     void* stream) {
  if (int rc = check_row_call(logits, dtype, N, V, ld, k, V < OPD_K_MAX ? V : OPD_K_MAX)) return rc;
  if (N == 0) return OPD_OK;
  if (!logits || !idx) return OPD_ERR_NULL;
  opd::CacheArgs a = row_args(logits, dtype, N, V, ld, k, mask, logp, lse_out);
  a.ids_out = idx;
  const hipError_t err = launch_cache_chunks(a, opd::CacheOp::Topk, dtype, row_fits(a.nvec, dtype),
                                           (hipStream_t)stream);
  return err == hipSuccess ? OPD_OK : OPD_ERR_HIP;
}

int opd_score_actions(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t ld,
                      const int32_t* ids, int32_t K, const uint8_t* mask, float* logp,
                      float* lse_out, void* stream) {
  if (int rc = check_row_call(logits, dtype, N, V, ld, K, OPD_K_MAX)) return rc;
  if (N == 0) return OPD_OK;
  if (!logits || !ids || !logp) return OPD_ERR_NULL;
  opd::CacheArgs a = row_args(logits, dtype, N, V, ld, K, mask, logp, lse_out);
  a.ids = ids;
  const hipError_t err = launch_cache_chunks(a, opd::CacheOp::Score, dtype, row_fits(a.nvec, dtype),
                                           (hipStream_t)stream);
  return err == hipSuccess ? OPD_OK : OPD_ERR_HIP;
}

int opd_quantize_blocks(const void* x, int32_t dtype, int64_t N, int64_t H, int64_t ldx,
                        int32_t block_rows, int32_t scale_type, void* q, int64_t ldq,
                        void* scales, void* stream) {
  if (dtype != OPD_F32 && dtype != OPD_BF16) return OPD_ERR_DTYPE;
  if (int rc = check_blocks(N, H, scale_type)) return rc;
  if (ldx < H || ldq < H) return OPD_ERR_SHAPE;
  if (block_rows != 1 && block_rows != 128) return OPD_ERR_PARAM;
  if (N == 0) return OPD_OK;
  if (!x || !q || !scales) return OPD_ERR_NULL;
  if (!aligned16(x) || !aligned16(q)) return OPD_ERR_ALIGN;
  if ((ldx * elt_bytes(dtype)) % 16 != 0 || ldq % 16 != 0) return OPD_ERR_ALIGN;
  if (scale_type == OPD_SCALE_F32 && !aligned4(scales)) return OPD_ERR_ALIGN;
  opd::QuantArgs a{};
  a.x = x;
  a.N = N;
  a.H = H;
  a.ldx = ldx;
  a.nb = (H + 127) / 128;
  a.block_rows = block_rows;
  a.q = (uint8_t*)q;
  a.ldq = ldq;
  a.scales = scales;
  const hipError_t err =
      opd::launch_quantize(a, dtype, scale_type == OPD_SCALE_E8M0, (hipStream_t)stream);
  return err == hipSuccess ? OPD_OK : OPD_ERR_HIP;
}

int opd_head_logits(const void* x, int64_t ldx, const void* x_scales, const void* w, int64_t ldw,
                    const void* w_scales, int32_t scale_type, int64_t N, int64_t V, int64_t H,
                    int32_t logits_dtype, void* logits, int64_t ld, void* stream) {
  if (logits_dtype != OPD_F32 && logits_dtype != OPD_BF16) return OPD_ERR_DTYPE;
  if (int rc = check_blocks(N, H, scale_type)) return rc;
  if (int rc = check_shape(N, V, ld)) return rc;
  if (V > kMaxHeadRows || ldx < H || ldw < H || ldx > kMaxHidden || ldw > kMaxHidden)
    return OPD_ERR_SHAPE;
  if (N * V > kMaxLogits) return OPD_ERR_SHAPE;
  if (N == 0) return OPD_OK;
  if (!x || !x_scales || !w || !w_scales || !logits) return OPD_ERR_NULL;
  if (!aligned16(x) || !aligned16(w) || !aligned16(logits)) return OPD_ERR_ALIGN;
  if (ldx % 16 != 0 || ldw % 16 != 0 || (ld * elt_bytes(logits_dtype)) % 16 != 0)
    return OPD_ERR_ALIGN;
  if (scale_type == OPD_SCALE_F32 && (!aligned4(x_scales) || !aligned4(w_scales)))
    return OPD_ERR_ALIGN;
  opd::HeadArgs a{};
  a.x = (const uint8_t*)x;
  a.sx = x_scales;
  a.w = (const uint8_t*)w;
  a.sw = w_scales;
  a.ldx = ldx;
  a.ldw = ldw;
  a.N = N;
  a.V = V;
  a.H = H;
  a.nb = (int)((H + 127) / 128);
  a.out = logits;
  a.ldo = ld;
  const hipError_t err =
      opd::launch_head(a, logits_dtype, scale_type == OPD_SCALE_E8M0, (hipStream_t)stream);
  return err == hipSuccess ? OPD_OK : OPD_ERR_HIP;
}

size_t opd_verify_workspace_bytes(int64_t B, int32_t D, int64_t V, int32_t dtype) {
  if (check_verify(dtype, B, D, V, V, V) != OPD_OK || B == 0) return 0;
  return (verify_plan(B, D, V, dtype, true).ws_bytes + 255) & ~(size_t)255;
}

int opd_verify_drafts(const void* target_logits, const void* draft_logits, int32_t dtype,
                      int64_t B, int32_t D, int64_t V, int64_t ld, int64_t draft_ld,
                      const int32_t* draft_ids, const int32_t* draft_lens, const float* uniforms,
                      const uint8_t* mask, int32_t* accepted, int32_t* ids, float* logp,
                      void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check_verify(dtype, B, D, V, ld, draft_logits ? draft_ld : V)) return rc;
  if (B == 0) return OPD_OK;
  if (!target_logits || !draft_ids || !uniforms || !accepted || !ids) return OPD_ERR_NULL;
  if (!aligned16(target_logits) || (ld * elt_bytes(dtype)) % 16 != 0) return OPD_ERR_ALIGN;
  if (draft_logits && (!aligned16(draft_logits) || (draft_ld * elt_bytes(dtype)) % 16 != 0))
    return OPD_ERR_ALIGN;
  if (!workspace || workspace_bytes < opd_verify_workspace_bytes(B, D, V, dtype) ||
      !aligned16(workspace))
    return OPD_ERR_WORKSPACE;
  opd::VerifyArgs a{};
  a.target = target_logits;
  a.draft = draft_logits;
  a.B = B;
  a.V = V;
  a.ld = ld;
  a.ldd = draft_ld;
  a.D = D;
  a.ids = draft_ids;
  a.lens = draft_lens;
  a.u = uniforms;
  a.mask = mask;
  a.accepted = accepted;
  a.ids_out = ids;
  a.logp = logp;
  const VerifyPlan p = verify_plan(B, D, V, dtype, draft_logits != nullptr);
  a.ws = workspace;
  a.parts = p.parts;
  a.part_groups = p.part_groups;
  a.draw_parts = p.draw_parts;
  a.nchunk = p.nchunk;
  a.chunk_steps = p.chunk_steps;
  a.table = p.table;
  a.round = p.round;
  const hipError_t err = opd::launch_verify(a, dtype, (hipStream_t)stream);
  return err == hipSuccess ? OPD_OK : OPD_ERR_HIP;
}

int opd_embed_tokens(const void* table, int32_t dtype, int64_t V, int64_t H, int64_t ld,
                     const int32_t* ids, int64_t N, float scale, void* out, int32_t out_dtype,
                     int64_t ldo, void* stream) {
  if (int rc = check_embed(dtype, out_dtype, N, V, H)) return rc;
  if (ld < H || ldo < H) return OPD_ERR_SHAPE;
  if (N == 0) return OPD_OK;
  if (!table || !ids || !out) return OPD_ERR_NULL;
  if (!rows_aligned(table, ld, dtype) || !rows_aligned(out, ldo, out_dtype)) return OPD_ERR_ALIGN;
  opd::EmbedArgs a{};
  a.table = table;
  a.V = V;
  a.H = H;
  a.ld = ld;
  a.ids = ids;
  a.N = N;
  a.scale = scale;
  a.out = out;
  a.ldo = ldo;
  const hipError_t err = opd::launch_embed(a, dtype, out_dtype, (hipStream_t)stream);
  return err == hipSuccess ? OPD_OK : OPD_ERR_HIP;
}

size_t opd_embed_workspace_bytes(int64_t N, int64_t V, int64_t H) {
  if (check_embed(OPD_F32, OPD_F32, N, V, H) != OPD_OK) return 0;
  return embed_layout(N, V, H).total;
}

int opd_embed_grads(const void* dy, int32_t dtype, int64_t N, int64_t H, int64_t ldy,
                    const int32_t* ids, int64_t V, float scale, void* dtable, int32_t out_dtype,
                    int64_t ldo, int32_t accumulate, void* workspace, size_t workspace_bytes,
                    void* stream) {
  if (int rc = check_embed(dtype, out_dtype, N, V, H)) return rc;
  if (ldy < H || ldo < H) return OPD_ERR_SHAPE;
  if (accumulate != 0 && accumulate != 1) return OPD_ERR_PARAM;
  if (!dtable || (N > 0 && (!dy || !ids))) return OPD_ERR_NULL;
  if (!rows_aligned(dtable, ldo, out_dtype) || (N > 0 && !rows_aligned(dy, ldy, dtype)))
    return OPD_ERR_ALIGN;
  // (one launch sorts, a workgroup to embed_keys(V) entries)
  if (!embed_unsorted(N, V, H) && (V + embed_keys(V) - 1) / embed_keys(V) * 1024 > kMaxGridLanes)
    return OPD_ERR_SHAPE;
  const EmbedLayout l = embed_layout(N, V, H);
  if (l.total > 0 && (!workspace || workspace_bytes < l.total || !aligned16(workspace)))
    return OPD_ERR_WORKSPACE;
  if (N == 0 && accumulate) return OPD_OK;
  opd::EmbedGradArgs a{};
  a.dy = dy;
  a.V = V;
  a.H = H;
  a.ldy = ldy;
  a.ids = ids;
  a.N = N;
  a.scale = scale;
  a.accumulate = accumulate;
  a.out = dtable;
  a.ldo = ldo;
  a.keys = embed_keys(V);
  char* ws = (char*)workspace;
  if (l.total > 0) {
    a.start = (int32_t*)ws;
    a.perm = (int32_t*)(ws + l.perm);
    a.partial = (float*)(ws + l.partial);
  }
  a.hp = l.hp;
  const hipError_t err = opd::launch_embed_grad(a, dtype, out_dtype, (hipStream_t)stream);
  return err == hipSuccess ? OPD_OK : OPD_ERR_HIP;
}

size_t opd_adapter_workspace_bytes(int64_t N, int64_t H, int64_t O, int32_t G, int32_t r,
                                   int32_t dtype, int32_t y_dtype, int32_t backward) {
  if (check_adapters(dtype, y_dtype, N, H, O, G, r) != OPD_OK) return 0;
  return adapt_layout(N, H, O, G, r, dtype, y_dtype, backward != 0).total;
}

int opd_add_adapters(const void* y, int32_t y_dtype, int64_t ldy, const void* x, int32_t dtype,
                     int64_t ldx, const void* a, int64_t lda, const void* b, int64_t ldb,
                     const float* scales, const int32_t* adapter_ids, int64_t N, int64_t H,
                     int64_t O, int32_t G, int32_t r, void* out, int64_t ldo, float* low_out,
                     void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check_adapters(dtype, y_dtype, N, H, O, G, r)) return rc;
  if (ldy < O || ldx < H || lda < H || ldb < O || ldo < O || lda > kMaxHidden || ldb > kMaxHidden)
    return OPD_ERR_SHAPE;
  if (N == 0) return OPD_OK;
  if (!y || !x || !a || !b || !adapter_ids || !out) return OPD_ERR_NULL;
  if (!rows_aligned(y, ldy, y_dtype) || !rows_aligned(out, ldo, y_dtype) ||
      !rows_aligned(x, ldx, dtype) || !rows_aligned(a, lda, dtype) || !rows_aligned(b, ldb, dtype))
    return OPD_ERR_ALIGN;
  if (y == out && ldy != ldo) return OPD_ERR_SHAPE;
  const AdaptLayout l = adapt_layout(N, H, O, G, r, dtype, y_dtype, false);
  if (!adapt_fits(l, O, G, false)) return OPD_ERR_SHAPE;
  if (!workspace || workspace_bytes < l.total || !aligned16(workspace)) return OPD_ERR_WORKSPACE;
  char* ws = (char*)workspace;
  const hipStream_t st = (hipStream_t)stream;
  const opd::AdaptArgs plan{adapter_ids, N, G, (int32_t*)ws, nullptr,
                            (opd::AdTile*)(ws + l.tiles), l.max_tiles};
  // (few tokens are grouped by the first product itself: a launch less)
  const bool few = N <= opd::kAdFew;
  hipError_t err = few ? hipSuccess : opd::launch_adapt_plan(plan, st);
  if (err != hipSuccess) return OPD_ERR_HIP;
  const opd::LowArgs t{plan.tiles, plan.perm, l.max_tiles, G, r, x, a, ldx, lda, H,
                       l.splits_x, l.span_x, N * l.ldt, (float*)(ws + l.t), l.ldt,
                       few ? adapter_ids : nullptr, (int)N};
  err = opd::launch_low(opd::LowPair{{t, {}}}, dtype, dtype, st);
  if (err != hipSuccess) return OPD_ERR_HIP;
  const opd::ExpandArgs e{plan.tiles, plan.perm, l.max_tiles, G, r,
                          opd::LowRef{t.out, t.ldo, t.stride, t.splits, r}, scales, b, ldb, O, y,
                          ldy, out, ldo, low_out, 0};
  err = opd::launch_expand(e, N, dtype, y_dtype, st);
  return err == hipSuccess ? OPD_OK : OPD_ERR_HIP;
}

int opd_adapter_grads(const void* dy, int32_t y_dtype, int64_t lddy, const void* x, int32_t dtype,
                      int64_t ldx, const void* a, int64_t lda, const void* b, int64_t ldb,
                      const float* scales, const int32_t* adapter_ids, int64_t N, int64_t H,
                      int64_t O, int32_t G, int32_t r, const float* low, const void* dx_shared,
                      int64_t ldds, void* dx, int64_t lddx, float* da, int64_t ldda, float* db,
                      int64_t lddb, void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check_adapters(dtype, y_dtype, N, H, O, G, r)) return rc;
  if (lddy < O || ldx < H || lda < H || ldb < O || ldda < H || lddb < O || (dx && lddx < H) ||
      (dx_shared && ldds < H) || lda > kMaxHidden || ldb > kMaxHidden)
    return OPD_ERR_SHAPE;
  if (!da || !db || !a || !b) return OPD_ERR_NULL;
  if (N > 0 && (!dy || !x || !adapter_ids || (dx_shared && !dx))) return OPD_ERR_NULL;
  if (!rows_aligned(a, lda, dtype) || !rows_aligned(b, ldb, dtype) ||
      !rows_aligned(da, ldda, OPD_F32) || !rows_aligned(db, lddb, OPD_F32))
    return OPD_ERR_ALIGN;
  if (N > 0 && (!rows_aligned(dy, lddy, y_dtype) || !rows_aligned(x, ldx, dtype) ||
                (dx && !rows_aligned(dx, lddx, dtype)) ||
                (dx_shared && !rows_aligned(dx_shared, ldds, dtype))))
    return OPD_ERR_ALIGN;
  if (dx && dx == dx_shared && lddx != ldds) return OPD_ERR_SHAPE;
  const AdaptLayout l = adapt_layout(N, H, O, G, r, dtype, y_dtype, true);
  if (!adapt_fits(l, H > O ? H : O, G, true)) return OPD_ERR_SHAPE;
  if (!workspace || workspace_bytes < l.total || !aligned16(workspace)) return OPD_ERR_WORKSPACE;
  char* ws = (char*)workspace;
  const hipStream_t st = (hipStream_t)stream;
  const opd::AdaptArgs plan{adapter_ids, N, G, (int32_t*)ws, (int32_t*)(ws + l.start),
                            (opd::AdTile*)(ws + l.tiles), l.max_tiles};
  hipError_t err = opd::launch_adapt_plan(plan, st);
  if (err != hipSuccess) return OPD_ERR_HIP;
  const opd::LowArgs t{plan.tiles, plan.perm, l.max_tiles, G, r, x, a, ldx, lda, H,
                       l.splits_x, l.span_x, N * l.ldt, (float*)(ws + l.t), l.ldt, nullptr, 0};
  const opd::LowArgs u{plan.tiles, plan.perm, l.max_tiles, G, r, dy, b, lddy, ldb, O,
                       l.splits_y, l.span_y, N * l.ldt, (float*)(ws + l.u), l.ldt, nullptr, 0};
  const opd::LowRef uref{u.out, u.ldo, u.stride, 1, r};
  const opd::LowRef tref =
      low ? opd::LowRef{low, r, 0, 1, r} : opd::LowRef{t.out, t.ldo, t.stride, 1, r};
  if (N > 0) {
    // (both products in one launch where their operands are of the same types)
    opd::LowPair first{{u, {}}}, then{{t, {}}};
    if (!low && dtype == y_dtype) first.a[1] = t;
    err = opd::launch_low(first, y_dtype, dtype, st);
    if (err == hipSuccess) err = opd::launch_low_sum(first, N, st);
    if (err == hipSuccess && !low && dtype != y_dtype) {
      err = opd::launch_low(then, dtype, dtype, st);
      if (err == hipSuccess) err = opd::launch_low_sum(then, N, st);
    }
    if (err != hipSuccess) return OPD_ERR_HIP;
  }
  const int64_t hp = (H + 3) / 4 * 4, op = (O + 3) / 4 * 4, gr = (int64_t)G * r;
  const opd::OuterPair pair{
      {{plan.perm, plan.start, G, r, uref, scales, x, ldx, H, l.outer, gr * hp,
        (float*)(ws + l.part_x), hp, da, ldda, 0},
       {plan.perm, plan.start, G, r, tref, scales, dy, lddy, O, l.outer, gr * op,
        (float*)(ws + l.part_y), op, db, lddb, 0}},
      0};
  err = opd::launch_outer(pair, dtype, y_dtype, st);
  if (err != hipSuccess) return OPD_ERR_HIP;
  if (!dx || N == 0) return OPD_OK;
  const opd::ExpandArgs e{plan.tiles, plan.perm, l.max_tiles, G, r, uref, scales, a, lda, H,
                          dx_shared, ldds, dx, lddx, nullptr, 0};
  err = opd::launch_expand(e, N, dtype, dtype, st);
  return err == hipSuccess ? OPD_OK : OPD_ERR_HIP;
}

size_t opd_beam_workspace_bytes(int64_t B, int32_t W, int64_t V, int32_t dtype) {
  if (check_beams(dtype, B, W, V, V) != OPD_OK || B == 0) return 0;
  return beam_plan(B, W, V, dtype).total;
}

int opd_beam_select(const void* logits, int32_t dtype, int64_t B, int32_t W, int64_t V, int64_t ld,
                    const float* scores, const uint8_t* finished, int32_t k, float* out_scores,
                    int32_t* parents, int32_t* ids, void* workspace, size_t workspace_bytes,
                    void* stream) {
  if (int rc = check_beams(dtype, B, W, V, ld)) return rc;
  if (k < 1 || k > OPD_BEAM_MAX) return OPD_ERR_SUPPORT;
  if (B == 0) return OPD_OK;
  if (!logits || !scores || !out_scores || !parents || !ids) return OPD_ERR_NULL;
  if (!rows_aligned(logits, ld, dtype)) return OPD_ERR_ALIGN;
  const BeamPlan p = beam_plan(B, W, V, dtype);
  if (!workspace || workspace_bytes < p.total || !aligned16(workspace)) return OPD_ERR_WORKSPACE;
  opd::BeamArgs a{};
  a.logits = logits;
  a.B = B;
  a.V = V;
  a.ld = ld;
  a.W = W;
  a.k = k;
  a.scores = scores;
  a.finished = finished;
  a.slots = p.slots;
  a.parts = (uint32_t)p.parts;
  a.recs = workspace;
  a.cands = (uint64_t*)((char*)workspace + p.cands);
  a.out_scores = out_scores;
  a.parents = parents;
  a.ids = ids;
  const hipError_t err = opd::launch_beam(a, dtype, (hipStream_t)stream);
  return err == hipSuccess ? OPD_OK : OPD_ERR_HIP;
}

int opd_reorder_beams(const void* states, int64_t B, int32_t W, int64_t outer, int64_t inner_bytes,
                      int64_t stride, int64_t outer_stride, const int32_t* parents, int32_t k,
                      void* out, int64_t out_stride, int64_t out_outer_stride, void* stream) {
  if (W < 1 || W > OPD_BEAM_MAX || k < 1 || k > OPD_BEAM_MAX) return OPD_ERR_SUPPORT;
  constexpr int64_t most = (int64_t)1 << 40;
  if (B < 0 || B > INT32_MAX || outer < 0 || outer > INT32_MAX || inner_bytes < 0 ||
      inner_bytes > most)
    return OPD_ERR_SHAPE;
  // (slices of a state do not overlap each other, nor do states of `out`)
  if (B > 0 && outer > 0 && inner_bytes > 0 &&
      (stride < 0 || out_stride < 0 || (outer > 1 && (outer_stride < inner_bytes ||
                                                      out_outer_stride < inner_bytes))))
    return OPD_ERR_SHAPE;
  if (B == 0 || outer == 0 || inner_bytes == 0) return OPD_OK;
  // states of `out` lie one after the other, or their slices do, a slice of all states
  // after the other
  const __int128 n = (__int128)B * k, gap = out_outer_stride;
  const bool whole = n == 1 || out_stride >= (outer - 1) * gap + inner_bytes;
  const bool sliced = outer == 1 || gap >= (n - 1) * (__int128)out_stride + inner_bytes;
  if (!whole && !(sliced && out_stride >= inner_bytes)) return OPD_ERR_SHAPE;
  if (!states || !parents || !out) return OPD_ERR_NULL;
  const bool in_place = states == out;
  if (in_place && (k != W || stride != out_stride || (outer > 1 && outer_stride != out_outer_stride)))
    return OPD_ERR_SHAPE;
  const opd::ReorderArgs a{states, B, W, k, outer, inner_bytes, stride, outer_stride, parents, out,
                           out_stride, out_outer_stride, in_place ? 1 : 0, 0, 0, 0};
  const hipError_t err = opd::launch_reorder(a, (hipStream_t)stream);
  return err == hipSuccess ? OPD_OK : OPD_ERR_HIP;
}

size_t opd_mc_diag_workspace_bytes(int64_t N, int32_t M, const int32_t* group_sizes,
                                   int32_t n_groups, int64_t seq_len) {
  if (check_diag(N, M, 0.5f, 0.2f, group_sizes, n_groups, seq_len) != OPD_OK) return 0;
  return diag_layout(N, M, n_groups, seq_len).total;
}

int opd_mc_diagnostics(const float* lse, const float* gathered, const float* teacher_logp,
                       const float* behav_logp, int64_t N, int32_t M, const uint8_t* mask,
                       float quantile, float clip_eps, const int32_t* group_sizes,
                       int32_t n_groups, int64_t seq_len, const opd_mc_diag* out, void* workspace,
                       size_t workspace_bytes, void* stream) {
  if (int rc = check_diag(N, M, quantile, clip_eps, group_sizes, n_groups, seq_len)) return rc;
  if (!out) return OPD_ERR_NULL;
  if (out->ratio_seq && (seq_len == 0 || n_groups == 0)) return OPD_ERR_PARAM;
  if (N == 0) return OPD_OK;
  if (!lse || !gathered || !teacher_logp || !behav_logp) return OPD_ERR_NULL;
  const DiagLayout l = diag_layout(N, M, n_groups, seq_len);
  if (!workspace || workspace_bytes < l.total || !aligned16(workspace)) return OPD_ERR_WORKSPACE;
  opd::DiagArgs a{};
  a.lse = lse;
  a.gathered = gathered;
  a.tau = teacher_logp;
  a.beta = behav_logp;
  a.N = N;
  a.M = M;
  a.mask = mask;
  a.q = quantile;
  a.clip_eps = clip_eps;
  a.n_groups = n_groups;
  for (int k = 0; k < n_groups; ++k) a.group[k] = group_sizes[k];
  a.seq_len = seq_len;
  a.nseq = l.nseq;
  a.pieces = l.pieces;
  a.row_mean = out->row_mean;
  a.row_var = out->row_var;
  a.row_rho_max = out->row_rho_max;
  a.rho_quantile = out->rho_quantile;
  a.clip_frac = out->clip_frac;
  a.ratio_local = out->ratio_local;
  a.ratio_seq = out->ratio_seq;
  char* ws = (char*)workspace;
  a.ws_rho = (uint32_t*)(ws + l.rho);
  a.ws_x = l.nseq && out->ratio_seq ? (float*)(ws + l.x) : nullptr;
  a.ws_psum = a.ws_x && l.pieces > 0 ? (double*)(ws + l.psum) : nullptr;
  a.ws_seq = a.ws_x ? (double*)(ws + l.seq) : nullptr;
  a.seq_groups = l.seq_groups;
  a.seq_batch = opd::diag_seq_batch(M, n_groups);
  a.ws_parts = (double*)(ws + l.parts);
  a.ws_hist = (uint32_t*)(ws + l.hist);
  const hipError_t err = opd::launch_diag(a, (hipStream_t)stream);
  return err == hipSuccess ? OPD_OK : OPD_ERR_HIP;
}

}  // extern "C"
